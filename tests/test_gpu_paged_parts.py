"""Selections whose workspace holds some of the rows only: the rows are taken in
parts, whose borders cut tiles of rows that share a slot."""
import numpy as np
import pytest

from gpu_common import require_gpu
from paper_2609_01068_amd import binding as B
from test_gpu_paged import cache_over, i32, plain_select, randn, scattered

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("width", [190, 1100])          # the fused form; the split form
@pytest.mark.parametrize("G", [1, 4])                   # tiles of 16 rows and of 4
@pytest.mark.parametrize("rows", [1, 4, 5, 20])
def test_parts_of_a_workspace(monkeypatch, width, G, rows):
    from paper_2609_01068_amd import paged
    n_kv, hd, top_k, lens = 2, 64, 20, [16 * width - 50] * 3
    table, slots = scattered(lens, 3 * width + 9, width, 2)
    table[slots[0], 50:60] = -1
    keys = randn((3 * width + 9, n_kv, hd), "bf16", 3)
    kv = cache_over(table, 3 * width + 9, n_kv, hd, "bf16", block_keys=keys)
    rs = np.repeat(slots, 17).astype(np.int32)
    rs[40] = -1
    pos = np.arange(16 * width - 120, 16 * width - 120 + 51, dtype=np.int32)
    q = randn((51, n_kv * G, hd), "bf16", 4)
    want = plain_select(keys.double().cpu().numpy(), q.double().cpu().numpy(), table, rs, pos, n_kv, top_k, 1, 2)
    need = B.lib().outlets_block_select_workspace(kv._ref, rows)
    assert need * 51 == rows * B.lib().outlets_block_select_workspace(kv._ref, 51)
    for spare in (0, need // rows - 1):                 # part of another row changes nothing
        monkeypatch.setattr(paged, "_SELECT_WS", need + spare)
        assert np.array_equal(kv.select(q, i32(rs), i32(pos), top_k, 1, 2).cpu().numpy(), want)
