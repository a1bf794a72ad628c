"""Torch-facing wrappers of the paged-cache operators: page tables kept on the
GPU (``PageTables``) and a paged KV cache with sparse attention over its pages
(``PagedKV``).

A decode step over a batch::

    rows = tables.append(slots, new_tokens, n_rows)
    kv.write(rows.slot_map, k, v)
    sel = kv.select(q, rows.row_slot, rows.positions, top_k=64)
    out = kv.attend(q, rows.row_slot, rows.positions, sel)

Every argument of a call is on the GPU and nothing is read back, so the step
can be captured into a graph.  Workspaces and outputs that are not passed come
from torch's allocator, on the call's stream.  PyTorch is used for device
memory and streams only.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Dict, NamedTuple, Optional

import torch

from . import binding as B

PAGE = 16
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_FMT = {"f32": B.OUTLETS_FMT_F32, "bf16": B.OUTLETS_FMT_BF16}


class Rows(NamedTuple):
    """The rows that an append laid out (device int32; -1 behind the last row).
    status = (0 or an error code, rows, pages taken, free pages left)."""
    cu: torch.Tensor
    slot_map: torch.Tensor
    positions: torch.Tensor
    row_slot: torch.Tensor
    status: torch.Tensor


def _take(buffers, name, shape, dtype, device, fill=None):
    """A buffer of the caller's, checked, or a new one."""
    t = (buffers or {}).get(name)
    if t is None:
        if fill is None:
            return torch.empty(shape, dtype=dtype, device=device)
        return torch.full(shape, fill, dtype=dtype, device=device)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check_i32(t, name, n, index):
    """Data pointer of a contiguous int32 vector (of n entries) on device `index`."""
    if t.dtype != torch.int32 or t.get_device() != index or t.dim() != 1 or not t.is_contiguous() or \
            (n is not None and t.shape[0] != n):
        raise TypeError(f"{name} must be a contiguous int32 tensor on cuda:{index}" +
                        ("" if n is None else f" of {n} entries"))
    return t.data_ptr()


_current_stream = torch._C._cuda_getCurrentRawStream     # (device index) -> handle, without a Stream object


def _on_stream(call):
    """A method that runs on its `stream` argument: what it allocates then
    belongs to that stream.  None is the current one."""
    @functools.wraps(call)
    def wrapper(self, *args, stream=None, **kw):
        if stream is None:
            return call(self, *args, **kw)
        if stream.device_index != self._index:
            raise ValueError(f"stream must be one of cuda:{self._index}")
        with torch.cuda.stream(stream):
            return call(self, *args, **kw)
    return wrapper


def _device(device) -> torch.device:
    d = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    return d if d.index is not None else torch.device("cuda", torch.cuda.current_device())


class PageTables:
    """Page tables of ``max_slots`` request slots over ``num_pages`` pages of 16
    tokens, kept on the GPU.

    ``buffers`` may hold the caller's own ``free_bits`` (int32
    [ceil(num_pages / 32)]), ``page_table`` (int32 [max_slots,
    ceil(max_seq_len / 16)]) and ``seq_len`` (int32 [max_slots]); given any, the
    state has only those, as they are (``append``, ``release`` and ``reset``
    need all three and are refused without), otherwise it starts empty."""

    def __init__(self, num_pages: int, max_slots: int, max_seq_len: int, device=0,
                 buffers: Optional[Dict[str, torch.Tensor]] = None):
        B.lib()
        self.device = _device(device)
        self._index = self.device.index
        self.num_pages, self.max_slots, self.max_seq_len = num_pages, max_slots, max_seq_len
        self.max_pages = -(-max_seq_len // PAGE)
        shapes = dict(free_bits=(-(-num_pages // 32),), page_table=(max_slots, self.max_pages), seq_len=(max_slots,))
        got = {name: _take(buffers, name, shape, torch.int32, self.device)
               if not buffers or buffers.get(name) is not None else None for name, shape in shapes.items()}
        self.free_bits, self.page_table, self.seq_len = got["free_bits"], got["page_table"], got["seq_len"]
        self._c = B.outlets_page_state(_ptr(self.free_bits), _ptr(self.page_table), _ptr(self.seq_len), num_pages,
                                       max_slots, max_seq_len, self.device.index)
        self._ref = C.byref(self._c)
        if not buffers:
            self.reset()

    @_on_stream
    def reset(self) -> None:
        B.check(B.lib().outlets_pages_reset(self._ref, _current_stream(self._index)), "outlets_pages_reset")

    @_on_stream
    def append(self, slots: torch.Tensor, new_tokens: torch.Tensor, n_rows: int, out: Optional[Rows] = None) -> Rows:
        """Append ``new_tokens[i]`` tokens to slot ``slots[i]`` (-1: padding) and
        lay out their rows, ``n_rows`` at most.  A refused call is reported in
        ``status[0]``, on the device."""
        n, lib = slots.shape[0], B.lib()
        sp, tp = _check_i32(slots, "slots", None, self._index), _check_i32(new_tokens, "new_tokens", n, self._index)
        if out is None:
            if n_rows < 0:
                raise ValueError("negative n_rows")
            buf = torch.empty(3 * n_rows + n + 5, dtype=torch.int32, device=self.device)
            sm, pos, rs, cu, status = buf.split_with_sizes((n_rows, n_rows, n_rows, n + 1, 4))
            out, base = Rows(cu, sm, pos, rs, status), buf.data_ptr()
            ptrs = (base + 12 * n_rows, base, base + 4 * n_rows, base + 8 * n_rows, base + 12 * n_rows + 4 * n + 4)
        else:
            ptrs = [_check_i32(t, name, m, self._index)
                    for t, name, m in zip(out, Rows._fields, (n + 1, n_rows, n_rows, n_rows, 4))]
        need = lib.outlets_pages_append_workspace(n, n_rows)
        ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        rc = lib.outlets_pages_append(self._ref, n, sp, tp, n_rows, *ptrs, ws.data_ptr() if need else None, need,
                                      _current_stream(self._index))
        if rc:
            B.check(rc, "outlets_pages_append")
        return out

    @_on_stream
    def release(self, slots: torch.Tensor) -> torch.Tensor:
        """Empty slots and free their pages; returns the device status word."""
        sp = _check_i32(slots, "slots", None, self._index)
        status = torch.empty(1, dtype=torch.int32, device=self.device)
        rc = B.lib().outlets_pages_release(self._ref, slots.shape[0], sp, status.data_ptr(), _current_stream(self._index))
        if rc:
            B.check(rc, "outlets_pages_release")
        return status


class PagedKV:
    """A paged KV cache over ``tables``: key pages [num_pages, n_kv, 16, hd],
    transposed value pages [num_pages, n_kv, hd, 16] and block keys [num_pages,
    n_kv, hd], in ``fmt`` ("f32" or "bf16").

    ``buffers`` may hold the caller's own ``k_pool``, ``v_pool`` and
    ``block_keys``; given any, the cache has only those (a call that needs
    another is refused)."""

    def __init__(self, tables: PageTables, n_kv: int, head_dim: int, fmt: str = "bf16",
                 buffers: Optional[Dict[str, torch.Tensor]] = None):
        self.tables, self.device, self._index = tables, tables.device, tables.device.index
        self.n_kv, self.head_dim, self.fmt, self.dtype = n_kv, head_dim, fmt, _DTYPES[fmt]
        p = tables.num_pages
        shapes = dict(k_pool=(p, n_kv, PAGE, head_dim), v_pool=(p, n_kv, head_dim, PAGE), block_keys=(p, n_kv, head_dim))
        got = {name: _take(buffers, name, shape, self.dtype, self.device) if not buffers or name in buffers else None
               for name, shape in shapes.items()}
        self.k_pool, self.v_pool, self.block_keys = got["k_pool"], got["v_pool"], got["block_keys"]
        self._c = B.outlets_kv_pages(_ptr(self.k_pool), _ptr(self.v_pool), _ptr(self.block_keys),
                                     _ptr(tables.page_table), _FMT[fmt], n_kv, head_dim, p, tables.max_slots,
                                     tables.max_pages, self.device.index)
        self._ref = C.byref(self._c)

    def _heads(self, t, name, n, heads):
        """Data pointer and row stride of rows [n, heads, hd], whose rows may stand apart."""
        hd = self.head_dim
        if t.dtype != self.dtype or t.get_device() != self._index or t.shape != (n, heads, hd):
            raise TypeError(f"{name} must be a {self.dtype} tensor of shape {(n, heads, hd)} on {self.device}")
        row, head, one = t.stride()
        if one != 1 or (heads > 1 and head != hd) or (n > 1 and row < heads * hd):
            raise ValueError(f"the heads of a row of {name} must stand together")
        return t.data_ptr(), row if n > 1 else max(row, heads * hd)

    @_on_stream
    def write(self, slot_map: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> None:
        """Store keys and values [n, n_kv, hd] of rows at ``slot_map`` (-1: skip)
        and the block keys of the pages that become full."""
        n = slot_map.shape[0]
        mp = _check_i32(slot_map, "slot_map", n, self._index)
        kp, ks = self._heads(k, "k", n, self.n_kv)
        vp, vs = self._heads(v, "v", n, self.n_kv)
        rc = B.lib().outlets_cache_write(self._ref, n, mp, kp, ks, vp, vs, _current_stream(self._index))
        if rc:
            B.check(rc, "outlets_cache_write")

    @_on_stream
    def select(self, q: torch.Tensor, row_slot: torch.Tensor, positions: torch.Tensor, top_k: int, sink: int = 1,
               local: int = 4, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Pages that each row's attention reads: int32 [n, n_kv, top_k]."""
        n, n_q = q.shape[0], q.shape[1]
        lib, index = B.lib(), self._index
        qp, qs = self._heads(q, "q", n, n_q)
        rp, pp = _check_i32(row_slot, "row_slot", n, index), _check_i32(positions, "positions", n, index)
        shape = (n, self.n_kv, top_k)
        if out is None:
            out = torch.empty(shape, dtype=torch.int32, device=self.device)
        elif out.shape != shape or out.dtype != torch.int32 or not out.is_contiguous() or out.get_device() != index:
            raise TypeError(f"out must be a contiguous int32 tensor of shape {shape} on {self.device}")
        need = 0
        if self.tables.max_pages > top_k and n:
            need = lib.outlets_block_select_workspace(self._ref, n)
            if need > _SELECT_WS:
                need = max(_SELECT_WS, lib.outlets_block_select_workspace(self._ref, 1))
        ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        rc = lib.outlets_block_select(self._ref, n, rp, pp, qp, qs, n_q, top_k, sink, local, out.data_ptr(),
                                      ws.data_ptr() if need else None, need, _current_stream(index))
        if rc:
            B.check(rc, "outlets_block_select")
        return out

    @_on_stream
    def attend(self, q: torch.Tensor, row_slot: torch.Tensor, positions: torch.Tensor, sel: torch.Tensor,
               gate: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention [n, n_q, hd] of each row over the pages of ``sel`` (as
        ``select`` gives them); ``out`` must not overlap ``q`` or ``gate``."""
        n, n_q = q.shape[0], q.shape[1]
        lib, index = B.lib(), self._index
        qp, qs = self._heads(q, "q", n, n_q)
        rp, pp = _check_i32(row_slot, "row_slot", n, index), _check_i32(positions, "positions", n, index)
        if sel.dim() != 3 or sel.shape[0] != n or sel.shape[1] != self.n_kv or sel.dtype != torch.int32 or \
                not sel.is_contiguous() or sel.get_device() != index:
            raise TypeError(f"sel must be a contiguous int32 tensor of shape ({n}, {self.n_kv}, top_k) on {self.device}")
        gp, gs = (None, 0) if gate is None else self._heads(gate, "gate", n, n_q)
        if out is None:
            out = torch.empty((n, n_q, self.head_dim), dtype=self.dtype, device=self.device)
            op, os_ = out.data_ptr(), n_q * self.head_dim
        else:
            op, os_ = self._heads(out, "out", n, n_q)
        need = lib.outlets_block_attention_workspace(self._ref, n, n_q, sel.shape[2])
        ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        rc = lib.outlets_block_attention(self._ref, n, rp, pp, qp, qs, n_q, sel.data_ptr(), sel.shape[2], gp, gs, op, os_,
                                         ws.data_ptr() if need else None, need, _current_stream(index))
        if rc:
            B.check(rc, "outlets_block_attention")
        return out


# Most bytes of scores that a selection holds at a time.
_SELECT_WS = 256 << 20
