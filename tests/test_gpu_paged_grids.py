"""Cache writes and page selections of more workgroups than one launch takes."""
import numpy as np
import pytest
import torch

from gpu_common import require_gpu
from test_gpu_paged import PAGE, cache_over, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def test_write_of_two_launches():
    """Pages whose rows lie on both sides of the border between two launches
    (2^21 rows of eight heads, unaligned rows)."""
    n, n_kv, hd, first = (1 << 21) + 5003, 8, 64, 5
    num = -(-(n + first) // PAGE) + 2
    kv = cache_over(np.zeros((1, 1), dtype=np.int32), num, n_kv, hd, "bf16",
                    **{name: torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for name, shape in
                       dict(k_pool=(num, n_kv, PAGE, hd), v_pool=(num, n_kv, hd, PAGE), block_keys=(num, n_kv, hd)).items()})
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    pages = torch.randperm(num, generator=g, device="cuda")
    at = torch.arange(first, first + n, device="cuda")
    page, off = pages[at // PAGE], at % PAGE
    wide = torch.empty((n, n_kv * hd + 1), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k = wide[:, 1:].view(n, n_kv, hd)
    kv.write((page * PAGE + off).int(), k, k)
    for r0 in range(0, n, 1 << 18):
        r = slice(r0, r0 + (1 << 18))
        assert torch.equal(kv.k_pool[page[r], :, off[r]], k[r])
        assert torch.equal(kv.v_pool[page[r], :, :, off[r]], k[r])
    full = page[off == PAGE - 1]
    for p0 in range(0, len(full), 1 << 14):
        p = full[p0:p0 + (1 << 14)]
        total = torch.zeros((len(p), n_kv, hd), dtype=torch.float64, device="cuda")
        for j in range(PAGE):
            total = total + kv.k_pool[p, :, j].double()
        assert torch.equal(kv.block_keys[p], (total / PAGE).float().bfloat16())
    left = pages[-2:]                                   # pages that no row names
    assert not kv.k_pool[left].any() and not kv.block_keys[left].any()


def test_write_of_very_many_heads():
    """65,535 heads, unaligned rows: 33 x 8 x 65,535 workgroups of 256 threads are more than 2^32 threads."""
    n, n_kv, hd, num = 4100, 65535, 64, 3
    kv = cache_over(np.zeros((1, 1), dtype=np.int32), num, n_kv, hd, "bf16",
                    **{name: torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for name, shape in
                       dict(k_pool=(num, n_kv, PAGE, hd), v_pool=(num, n_kv, hd, PAGE), block_keys=(num, n_kv, hd)).items()})
    k = torch.empty(n * n_kv * hd + 1, dtype=torch.bfloat16, device="cuda")[1:].view(n, n_kv, hd)   # (tiles of 16 rows)
    slot_map = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    ends = list(range(7)) + list(range(n - 25, n))      # page 2 from its tenth token on, then pages 0 and 1
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for i, r in enumerate(ends):
        k[r].normal_(generator=g)
        slot_map[r] = 2 * PAGE + 9 + i if i < 7 else i - 7
    kv.write(slot_map, k, k)
    for r in ends:
        s = int(slot_map[r])
        assert torch.equal(kv.k_pool[s // PAGE, :, s % PAGE], k[r])
        assert torch.equal(kv.v_pool[s // PAGE, :, :, s % PAGE], k[r])
    for p in (0, 2):                                    # page 2's first nine keys stand in the pool, zeros
        total = torch.zeros((n_kv, hd), dtype=torch.float64, device="cuda")
        for j in range(PAGE):
            total = total + kv.k_pool[p, :, j].double()
        assert torch.equal(kv.block_keys[p], (total / PAGE).float().bfloat16())
    assert not kv.block_keys[1].any() and not kv.k_pool[1, :, 9:].any() and not kv.k_pool[2, :, :9].any()


def test_select_of_many_rows_and_heads():
    """17,000 rows of 1,024 heads, all pages selected: more than 2^32 threads."""
    n, n_kv, hd = 17000, 1024, 64
    table = np.arange(6, dtype=np.int32).reshape(3, 2)
    kv = cache_over(table, 6, n_kv, hd, "bf16",
                    block_keys=torch.zeros((6, n_kv, hd), dtype=torch.bfloat16, device="cuda"))
    q = torch.zeros((n, n_kv, hd), dtype=torch.bfloat16, device="cuda")
    pos = np.arange(n, dtype=np.int32) % 33 - 1         # -1 .. 31
    sel = kv.select(q, i32(np.arange(n) % 3), i32(pos), 2, 0, 1)
    nb = torch.as_tensor((pos + 16) // 16, device="cuda")[:, None, None]
    want = torch.arange(2, device="cuda").expand(n, n_kv, 2)
    assert torch.equal(sel.long(), torch.where(want < nb, want, -1))
