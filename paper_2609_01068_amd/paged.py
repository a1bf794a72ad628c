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

import contextlib
import ctypes as C
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


def _check_i32(t, name, n, device):
    if t.dtype != torch.int32 or t.device != device or t.dim() != 1 or not t.is_contiguous() or (n is not None and len(t) != n):
        raise TypeError(f"{name} must be a contiguous int32 tensor on {device}" + ("" if n is None else f" of {n} entries"))
    return t.data_ptr()


@contextlib.contextmanager
def _on(device, stream):
    """The call's stream (its handle for the library); tensors that a call
    allocates belong to it."""
    if stream is None:
        yield torch.cuda.current_stream(device).cuda_stream or None
    else:
        with torch.cuda.stream(stream):
            yield stream.cuda_stream or None


def _device(device) -> torch.device:
    d = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    return d if d.index is not None else torch.device("cuda", torch.cuda.current_device())


class PageTables:
    """Page tables of ``max_slots`` request slots over ``num_pages`` pages of 16
    tokens, kept on the GPU.

    ``buffers`` may hold the caller's own ``free_bits`` (int32
    [ceil(num_pages / 32)]), ``page_table`` (int32 [max_slots,
    ceil(max_seq_len / 16)]) and ``seq_len`` (int32 [max_slots]); given any, all
    are taken as they are (``reset`` empties them), otherwise the state starts
    empty."""

    def __init__(self, num_pages: int, max_slots: int, max_seq_len: int, device=0,
                 buffers: Optional[Dict[str, torch.Tensor]] = None):
        B.lib()
        self.device = _device(device)
        self.num_pages, self.max_slots, self.max_seq_len = num_pages, max_slots, max_seq_len
        self.max_pages = -(-max_seq_len // PAGE)
        self.free_bits = _take(buffers, "free_bits", (-(-num_pages // 32),), torch.int32, self.device)
        self.page_table = _take(buffers, "page_table", (max_slots, self.max_pages), torch.int32, self.device)
        self.seq_len = _take(buffers, "seq_len", (max_slots,), torch.int32, self.device)
        self._c = B.outlets_page_state(self.free_bits.data_ptr(), self.page_table.data_ptr(), self.seq_len.data_ptr(),
                                       num_pages, max_slots, max_seq_len, self.device.index)
        self._ref = C.byref(self._c)
        if not buffers:
            self.reset()

    def reset(self, stream=None) -> None:
        with _on(self.device, stream) as st:
            B.check(B.lib().outlets_pages_reset(self._ref, st), "outlets_pages_reset")

    def append(self, slots: torch.Tensor, new_tokens: torch.Tensor, n_rows: int, out: Optional[Rows] = None,
               stream=None) -> Rows:
        """Append ``new_tokens[i]`` tokens to slot ``slots[i]`` (-1: padding) and
        lay out their rows, ``n_rows`` at most.  A refused call is reported in
        ``status[0]``, on the device."""
        n = len(slots)
        sp, tp = _check_i32(slots, "slots", None, self.device), _check_i32(new_tokens, "new_tokens", n, self.device)
        with _on(self.device, stream) as st:
            if out is None:
                # one allocation, sliced; every part 16 bytes apart or more
                a, r = -(-(n + 1) // 4) * 4, -(-n_rows // 4) * 4
                buf = torch.empty(a + 3 * r + 4, dtype=torch.int32, device=self.device)
                out = Rows(buf[:n + 1], buf[a:a + n_rows], buf[a + r:a + r + n_rows],
                           buf[a + 2 * r:a + 2 * r + n_rows], buf[a + 3 * r:])
            else:
                for t, name, m in zip(out, Rows._fields, (n + 1, n_rows, n_rows, n_rows, 4)):
                    _check_i32(t, name, m, self.device)
            need = B.lib().outlets_pages_append_workspace(n, n_rows)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            rc = B.lib().outlets_pages_append(self._ref, n, sp, tp, n_rows, out.cu.data_ptr(), out.slot_map.data_ptr(),
                                              out.positions.data_ptr(), out.row_slot.data_ptr(),
                                              out.status.data_ptr(), ws.data_ptr() if need else None, need, st)
        B.check(rc, "outlets_pages_append")
        return out

    def release(self, slots: torch.Tensor, stream=None) -> torch.Tensor:
        """Empty slots and free their pages; returns the device status word."""
        sp = _check_i32(slots, "slots", None, self.device)
        with _on(self.device, stream) as st:
            status = torch.empty(1, dtype=torch.int32, device=self.device)
            rc = B.lib().outlets_pages_release(self._ref, len(slots), sp, status.data_ptr(), st)
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
        self.tables, self.device = tables, tables.device
        self.n_kv, self.head_dim, self.fmt, self.dtype = n_kv, head_dim, fmt, _DTYPES[fmt]
        p = tables.num_pages
        shapes = dict(k_pool=(p, n_kv, PAGE, head_dim), v_pool=(p, n_kv, head_dim, PAGE), block_keys=(p, n_kv, head_dim))
        got = {name: _take(buffers, name, shape, self.dtype, self.device) if not buffers or name in buffers else None
               for name, shape in shapes.items()}
        self.k_pool, self.v_pool, self.block_keys = got["k_pool"], got["v_pool"], got["block_keys"]
        ptr = {name: None if t is None else t.data_ptr() for name, t in got.items()}
        self._c = B.outlets_kv_pages(ptr["k_pool"], ptr["v_pool"], ptr["block_keys"], tables.page_table.data_ptr(),
                                     _FMT[fmt], n_kv, head_dim, p, tables.max_slots, tables.max_pages,
                                     self.device.index)
        self._ref = C.byref(self._c)

    def _heads(self, t, name, n, heads):
        """Data pointer and row stride of rows [n, heads, hd], whose rows may stand apart."""
        if t.dtype != self.dtype or t.device != self.device or tuple(t.shape) != (n, heads, self.head_dim):
            raise TypeError(f"{name} must be a {self.dtype} tensor of shape {(n, heads, self.head_dim)} on {self.device}")
        row, head, one = t.stride()
        if one != 1 or (heads > 1 and head != self.head_dim) or (n > 1 and row < heads * self.head_dim):
            raise ValueError(f"the heads of a row of {name} must stand together")
        return t.data_ptr(), row if n > 1 else max(row, heads * self.head_dim)

    def write(self, slot_map: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Store keys and values [n, n_kv, hd] of rows at ``slot_map`` (-1: skip)
        and the block keys of the pages that become full."""
        n = len(slot_map)
        mp = _check_i32(slot_map, "slot_map", None, self.device)
        kp, ks = self._heads(k, "k", n, self.n_kv)
        vp, vs = self._heads(v, "v", n, self.n_kv)
        with _on(self.device, stream) as st:
            rc = B.lib().outlets_cache_write(self._ref, n, mp, kp, ks, vp, vs, st)
        B.check(rc, "outlets_cache_write")

    def select(self, q: torch.Tensor, row_slot: torch.Tensor, positions: torch.Tensor, top_k: int, sink: int = 1,
               local: int = 4, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Pages that each row's attention reads: int32 [n, n_kv, top_k]."""
        n, n_q = q.shape[0], q.shape[1]
        qp, qs = self._heads(q, "q", n, n_q)
        rp, pp = _check_i32(row_slot, "row_slot", n, self.device), _check_i32(positions, "positions", n, self.device)
        with _on(self.device, stream) as st:
            shape = (n, self.n_kv, top_k)
            if out is None:
                out = torch.empty(shape, dtype=torch.int32, device=self.device)
            elif tuple(out.shape) != shape or out.dtype != torch.int32 or not out.is_contiguous() or out.device != self.device:
                raise TypeError(f"out must be a contiguous int32 tensor of shape {shape} on {self.device}")
            need = 0
            if self.tables.max_pages > top_k and n:
                need = B.lib().outlets_block_select_workspace(self._ref, n)
                if need > _SELECT_WS:
                    need = max(_SELECT_WS, B.lib().outlets_block_select_workspace(self._ref, 1))
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            rc = B.lib().outlets_block_select(self._ref, n, rp, pp, qp, qs, n_q, top_k, sink, local, out.data_ptr(),
                                              ws.data_ptr() if need else None, need, st)
        B.check(rc, "outlets_block_select")
        return out

    def attend(self, q: torch.Tensor, row_slot: torch.Tensor, positions: torch.Tensor, sel: torch.Tensor,
               gate: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention [n, n_q, hd] of each row over the pages of ``sel`` (as ``select`` gives them)."""
        n, n_q = q.shape[0], q.shape[1]
        qp, qs = self._heads(q, "q", n, n_q)
        rp, pp = _check_i32(row_slot, "row_slot", n, self.device), _check_i32(positions, "positions", n, self.device)
        if sel.dim() != 3 or tuple(sel.shape[:2]) != (n, self.n_kv) or sel.dtype != torch.int32 or \
                not sel.is_contiguous() or sel.device != self.device:
            raise TypeError(f"sel must be a contiguous int32 tensor of shape ({n}, {self.n_kv}, top_k) on {self.device}")
        gp, gs = (None, 0) if gate is None else self._heads(gate, "gate", n, n_q)
        with _on(self.device, stream) as st:
            if out is None:
                out = torch.empty((n, n_q, self.head_dim), dtype=self.dtype, device=self.device)
            op, os_ = self._heads(out, "out", n, n_q)
            need = B.lib().outlets_block_attention_workspace(self._ref, n, n_q, sel.shape[2])
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            rc = B.lib().outlets_block_attention(self._ref, n, rp, pp, qp, qs, n_q, sel.data_ptr(), sel.shape[2], gp, gs,
                                                 op, os_, ws.data_ptr() if need else None, need, st)
        B.check(rc, "outlets_block_attention")
        return out


# Most bytes of scores that a selection holds at a time.
_SELECT_WS = 256 << 20
