"""Sums of the attention over selected pages (bf16): how exact the softmax
weights are, infinite values, and the same bits from call to call.

Tolerance, in the terms of test_gpu_paged.py: a weight enters the second
product as two bf16 values, the second of the first one's error, so it is off by
at most 2^-8 2^-8 of itself, and the row sum adds the weight itself: the output
moves by at most 2^-16 (A + |o|) instead of 2^-8 A.
"""
import numpy as np
import pytest
import torch

from gpu_common import require_gpu
from test_gpu_paged import attention_ref, cache_over, fill_pages, i32, randn, scattered

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def rows_of(kind, n_kv, top_k, seed):
    """(row slots' indexes, positions, selections): rows of their own slots, a
    prompt's rows, or few rows of many pages (split)."""
    r = np.random.default_rng(seed)
    n = {"own": 150, "shared": 300, "split": 3}[kind]
    which = np.arange(n) % 2 if kind != "shared" else np.repeat([0, 1], [n - 50, 50])
    pos = r.integers(1700, 2000, size=n) if kind != "shared" else 1600 + np.arange(n)
    sel = np.full((n, n_kv, top_k), -1, dtype=np.int32)
    for i in range(n):
        for g in range(n_kv):
            sel[i, g] = np.sort(r.permutation(pos[i] // PAGE + 1)[:top_k])
    return which, pos.astype(np.int32), sel


@pytest.mark.parametrize("hd,n_kv,G", [(128, 2, 4), (64, 2, 2), (128, 1, 16)])
@pytest.mark.parametrize("kind", ["own", "shared", "split"])
@pytest.mark.parametrize("gated", [False, True])
def test_weights_of_sixteen_bits(hd, n_kv, G, kind, gated):
    top_k = 70
    lens = [2000, 2000]
    table, slots = scattered(lens, 260, 130, 5)
    k, v = fill_pages(table, lens, slots, 260, n_kv, hd, "bf16")
    kv = cache_over(table, 260, n_kv, hd, "bf16", k_pool=k, v_pool=v)
    which, pos, sel = rows_of(kind, n_kv, top_k, hd + G)
    rs = slots[which].astype(np.int32)
    q = randn((len(pos), n_kv * G, hd), "bf16", 6)
    gate = randn(q.shape, "bf16", 7) if gated else None
    got = f64(kv.attend(q, i32(rs), i32(pos), i32(sel), gate=gate))
    ref, e32, e16 = attention_ref(f64(k), f64(v), f64(q), table, rs, pos, sel, f64(gate))
    tol = 1.01 * (e32 + 2.0**-8 * e16 + 2.0**-16 * np.abs(ref) + 2.0**-8 * np.abs(ref))
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()


@pytest.mark.parametrize("kind", ["own", "shared", "split"])
def test_infinite_values(kind):
    """An infinite value of a page that a row reads makes its channel infinite,
    with its sign, whatever the weight's second part; the other channels are
    those of weights of eight bits at least."""
    hd, n_kv, G, top_k = 128, 2, 4, 40
    lens = [2000, 2000]
    table, slots = scattered(lens, 260, 130, 5)
    k, v = fill_pages(table, lens, slots, 260, n_kv, hd, "bf16")
    for page in range(0, 100, 7):
        v[table[slots[0], page], :, 5, page % PAGE] = float("inf")
        v[table[slots[1], page], :, 77, 3] = float("-inf")
    kv = cache_over(table, 260, n_kv, hd, "bf16", k_pool=k, v_pool=v)
    which, pos, sel = rows_of(kind, n_kv, top_k, 3)
    rs = slots[which].astype(np.int32)
    q = randn((len(pos), n_kv * G, hd), "bf16", 6)
    got = f64(kv.attend(q, i32(rs), i32(pos), i32(sel)))
    with np.errstate(invalid="ignore"):
        ref, e32, e16 = attention_ref(f64(k), f64(v), f64(q), table, rs, pos, sel, None)
    inf = np.isinf(ref)
    assert inf.any() and not np.isnan(ref).any() and np.array_equal(got[inf], ref[inf])
    tol = 1.01 * (e32 + e16 + 2.0**-8 * np.abs(ref))
    assert (np.abs(got[~inf] - ref[~inf]) <= tol[~inf]).all()


@pytest.mark.parametrize("hd,G", [(128, 4), (64, 2), (128, 1)])
def test_calls_repeat_their_bits(hd, G):
    """Rows that share pages, whose lists name them in any order: the same call
    again, with other work before it, and with its lists in another order."""
    n_kv, top_k, lens = 8, 96, [5000, 5000, 5000, 5000]
    table, slots = scattered(lens, 1300, 320, 5)
    k, v = fill_pages(table, lens, slots, 1300, n_kv, hd, "bf16")
    kv = cache_over(table, 1300, n_kv, hd, "bf16", k_pool=k, v_pool=v)
    n = 440
    rs = i32(slots[np.arange(n) // 110])
    pos = i32(4500 + np.arange(n))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    order = torch.rand((n, n_kv, 280), generator=g, device="cuda").argsort(dim=2).to(torch.int32)
    sel = order[..., :top_k].contiguous()
    q = randn((n, n_kv * G, hd), "bf16", 6)
    lists = [sel, sel.sort(dim=2).values]
    first = [kv.attend(q, rs, pos, x).view(torch.int16) for x in lists]
    # rows taken together (16 / G of one slot) read the pages in their order,
    # single rows in that of their list
    i = np.arange(n)
    r0 = i // (16 // G) * (16 // G)
    together = torch.as_tensor(r0 // 110 == np.minimum(r0 + 16 // G, n) // 110, device="cuda")
    assert torch.equal(first[0][together], first[1][together])
    for turn in range(30):
        if turn % 3 == 1:
            torch.randn((2000, 2000), device="cuda").sort(dim=0)
        again = kv.attend(q, rs, pos, lists[turn % 2])
        assert torch.equal(first[turn % 2], again.view(torch.int16)), turn
