"""PageTables over some of the caller's buffers: calls that need a missing part
are refused before any device work, so host memory stands in for the device's."""
import itertools

import pytest
import torch

from paper_2609_01068_amd import binding as B
from test_gemm_dispatch import library_host

NAMES = dict(free_bits=(2,), page_table=(4, 3), seq_len=(4,))


@pytest.fixture(autouse=True)
def _host_memory(monkeypatch):
    library_host()          # builds a missing library
    from paper_2609_01068_amd import paged

    class Device:           # a device of index 0 that torch allocates host memory for
        index = 0
    monkeypatch.setattr(paged, "_device", lambda d: Device())
    monkeypatch.setattr(paged, "_current_stream", lambda index: None)
    monkeypatch.setattr(paged, "_check_i32", lambda t, name, n, index: t.data_ptr())
    monkeypatch.setattr(paged, "_take", lambda buffers, name, shape, dtype, device:
                        (buffers or {}).get(name) if (buffers or {}).get(name) is not None
                        else torch.empty(shape, dtype=dtype))
    empty = torch.empty
    monkeypatch.setattr(paged.torch, "empty", lambda *a, **kw: empty(*a, **{**kw, "device": "cpu"}))


@pytest.mark.parametrize("given", [c for k in (1, 2) for c in itertools.combinations(NAMES, k)])
@pytest.mark.parametrize("spelled", [False, True])      # the others left out, or None
def test_missing_page_state_is_refused(given, spelled):
    from paper_2609_01068_amd.paged import PageTables
    buffers = {name: torch.zeros(NAMES[name], dtype=torch.int32) for name in given}
    if spelled:
        buffers.update({name: None for name in NAMES if name not in given})
    pt = PageTables(40, 4, 40, buffers=buffers)
    assert all((getattr(pt, name) is not None) == (name in given) for name in NAMES)
    slots = torch.zeros(1, dtype=torch.int32)
    for call in (pt.reset, lambda: pt.append(slots, slots, 4), lambda: pt.release(slots)):
        with pytest.raises(B.OutletsError) as e:
            call()
        assert e.value.rc == B.OUTLETS_ERR_INVALID_ARG and "null page state memory" in str(e.value)
    assert all((t == 0).all() for t in buffers.values() if t is not None)


def test_a_cache_without_a_page_table():
    from paper_2609_01068_amd.paged import PagedKV, PageTables
    pt = PageTables(40, 4, 40, buffers=dict(seq_len=torch.zeros(4, dtype=torch.int32)))
    kv = PagedKV(pt, 1, 64, "f32", buffers=dict(block_keys=torch.zeros(40, 1, 64)))
    q, rows = torch.zeros(1, 1, 64), torch.zeros(1, dtype=torch.int32)
    kv._heads = lambda t, name, n, heads: (t.data_ptr(), 64)
    with pytest.raises(B.OutletsError) as e:
        kv.select(q, rows, rows, 2, 0, 1, out=None)
    assert e.value.rc == B.OUTLETS_ERR_INVALID_ARG and "page table" in str(e.value)
