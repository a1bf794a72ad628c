"""Argument checks of the paged-cache operators: every refusal comes before
any device work, so it is the same without a GPU."""
import ctypes as C

import pytest

from paper_2609_01068_amd import binding as B

from test_gemm_dispatch import library_host


@pytest.fixture(scope="module", autouse=True)
def _library():
    library_host()          # builds a missing library


A = 0x10000      # a non-null, 16-byte aligned address that no refused call touches


def state(**kw):
    v = dict(free_bits=A, page_table=A, seq_len=A, num_pages=8, max_slots=4, max_seq_len=100, device=0)
    v.update(kw)
    return B.outlets_page_state(*[v[n] for n, _ in B.outlets_page_state._fields_])


def cache(**kw):
    v = dict(k_pool=A, v_pool=A, block_keys=A, page_table=A, fmt=B.OUTLETS_FMT_BF16, n_kv_heads=2, head_dim=128,
             num_pages=8, max_slots=4, max_pages=7, device=0)
    v.update(kw)
    return B.outlets_kv_pages(*[v[n] for n, _ in B.outlets_kv_pages._fields_])


def refused(rc, want):
    assert rc == want and B.last_error() != ""


INV, UNS = B.OUTLETS_ERR_INVALID_ARG, B.OUTLETS_ERR_UNSUPPORTED


def append(s, n=1, slots=A, new=A, rows=4, cu=A, sm=A, pos=A, rs=A, status=A, ws=None, ws_bytes=0):
    return B.lib().outlets_pages_append(C.byref(s) if s else None, n, slots, new, rows, cu, sm, pos, rs, status, ws,
                                        ws_bytes, None)


@pytest.mark.parametrize("bad,want", [
    (dict(num_pages=0), INV), (dict(num_pages=1 << 27), INV), (dict(max_slots=0), INV), (dict(max_seq_len=0), INV),
    (dict(max_seq_len=2**31 - 1), INV), (dict(max_slots=(1 << 17) + 1), UNS), (dict(device=-1), INV),
    (dict(free_bits=None), INV), (dict(page_table=None), INV), (dict(seq_len=None), INV)])
def test_page_state_refusals(bad, want):
    s = state(**bad)
    refused(append(s), want)
    refused(B.lib().outlets_pages_reset(C.byref(s), None), want)
    refused(B.lib().outlets_pages_release(C.byref(s), 1, A, A, None), want)


def test_page_call_refusals():
    refused(append(None), INV)
    s = state()
    refused(append(s, n=-1), INV)
    refused(append(s, rows=-1), INV)
    refused(append(s, rows=(1 << 20) + 1), UNS)
    refused(append(s, n=(1 << 20) + 1), UNS)
    for k in ("slots", "new", "cu", "sm", "pos", "rs", "status"):
        refused(append(s, **{k: None}), INV)
    need = B.lib().outlets_pages_append_workspace(3, 5000)
    assert need > 0 and B.lib().outlets_pages_append_workspace(512, 512) == 0
    refused(append(s, n=3, rows=5000), INV)
    refused(append(s, n=3, rows=5000, ws=A, ws_bytes=need - 1), INV)
    refused(append(s, n=3, rows=5000, ws=A + 4, ws_bytes=need), INV)
    r = B.lib().outlets_pages_release
    refused(r(C.byref(s), -1, A, A, None), INV)
    refused(r(C.byref(s), 1, None, A, None), INV)
    refused(r(C.byref(s), 1, A, None, None), INV)
    refused(r(C.byref(s), (1 << 18) + 1, A, A, None), UNS)


def write(c, n=1, sm=A, k=A, ks=256, v=A, vs=256):
    return B.lib().outlets_cache_write(C.byref(c) if c else None, n, sm, k, ks, v, vs, None)


def select(c, n=1, rs=A, pos=A, q=A, qs=1024, n_q=8, top_k=4, sink=1, local=1, sel=A, ws=A, ws_bytes=1 << 20):
    return B.lib().outlets_block_select(C.byref(c) if c else None, n, rs, pos, q, qs, n_q, top_k, sink, local, sel, ws,
                                        ws_bytes, None)


def attend(c, n=1, rs=A, pos=A, q=A, qs=1024, n_q=8, sel=A, top_k=4, gate=None, gs=0, out=A, os=1024, ws=A,
           ws_bytes=1 << 30):
    return B.lib().outlets_block_attention(C.byref(c) if c else None, n, rs, pos, q, qs, n_q, sel, top_k, gate, gs, out,
                                           os, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,want", [
    (dict(fmt=B.OUTLETS_FMT_E4M3), UNS), (dict(head_dim=96), UNS), (dict(n_kv_heads=0), INV),
    (dict(n_kv_heads=65536), INV), (dict(num_pages=0), INV), (dict(num_pages=1 << 27), INV), (dict(device=-1), INV),
    (dict(k_pool=A + 8), UNS), (dict(v_pool=A + 8), UNS), (dict(block_keys=A + 8), UNS)])
def test_cache_refusals(bad, want):
    c = cache(**bad)
    for call in (write, select, attend):
        refused(call(c), want)
    assert B.lib().outlets_block_select_workspace(C.byref(c), 4) == 0
    assert B.lib().outlets_block_attention_workspace(C.byref(c), 4, 8, 4) == 0


def test_call_refusals():
    for call in (write, select, attend):
        refused(call(None), INV)
        refused(call(cache(), n=-1), INV)
    c = cache()
    refused(write(cache(k_pool=None)), INV)
    refused(write(cache(v_pool=None)), INV)
    for k in ("sm", "k", "v"):
        refused(write(c, **{k: None}), INV)
    refused(write(c, ks=255), INV)
    refused(write(c, vs=255), INV)
    for call in (select, attend):
        refused(call(cache(page_table=None)), INV)
        refused(call(cache(max_slots=0)), INV)
        refused(call(cache(max_pages=0)), INV)
        refused(call(c, n_q=7), INV)
        refused(call(c, n_q=0), INV)
        refused(call(c, n_q=34, qs=34 * 128), UNS)
        refused(call(c, qs=1023), INV)
        refused(call(c, top_k=0), INV)
        for k in ("rs", "pos", "q", "sel"):
            refused(call(c, **{k: None}), INV)
    refused(select(cache(block_keys=None)), INV)
    refused(select(c, sink=-1), INV)
    refused(select(c, local=0), INV)
    refused(select(c, sink=2, local=3), INV)
    refused(select(c, sink=2**31 - 1, local=2**31 - 1), INV)
    one = B.lib().outlets_block_select_workspace(C.byref(c), 1)
    assert one > 0 and B.lib().outlets_block_select_workspace(C.byref(c), 5) == 5 * one
    refused(select(c, ws=None), INV)
    refused(select(c, ws_bytes=one - 1), INV)
    refused(select(c, ws=A + 8), INV)
    refused(attend(cache(k_pool=None)), INV)
    refused(attend(cache(v_pool=None)), INV)
    refused(attend(c, out=None), INV)
    refused(attend(c, os=1023), INV)
    refused(attend(c, gate=A, gs=1023), INV)
    refused(attend(c, q=A + 8), UNS)
    refused(attend(c, qs=1025), UNS)


def test_empty_calls_need_no_gpu():
    assert write(cache(), n=0, sm=None, k=None, v=None) == B.OUTLETS_OK
    assert select(cache(), n=0, rs=None, pos=None, q=None, sel=None, ws=None) == B.OUTLETS_OK
    assert attend(cache(), n=0, rs=None, pos=None, q=None, sel=None, out=None, ws=None) == B.OUTLETS_OK


def test_streams_of_other_devices_are_refused():
    """One that is not the tables' would leave the call on the current stream."""
    from paper_2609_01068_amd import paged

    class Stream:
        device_index = 1

    tables = object.__new__(paged.PageTables)
    tables._index = 0
    for call in (tables.reset, lambda **kw: tables.append(None, None, 1, **kw), lambda **kw: tables.release(None, **kw)):
        with pytest.raises(ValueError, match="cuda:0"):
            call(stream=Stream())
    kv = object.__new__(paged.PagedKV)
    kv._index = 0
    for call, n in ((kv.write, 3), (kv.select, 4), (kv.attend, 4)):
        with pytest.raises(ValueError, match="cuda:0"):
            call(*[None] * n, stream=Stream())
