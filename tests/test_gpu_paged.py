"""Paged-cache operators on the GPU against plain forms in 64 bits: page tables
(bit for bit with the host allocator), cache write, page selection (equal
index for index) and attention over selected pages.

Tolerances of the attention, per output element, with w the softmax weights, o
the output and A = sum_i w_i |v_i - o|:
- fp32 scores: a dot product of hd terms is off by at most (hd + 2) 2^-24
  sum |q k| scale, e say; weights off by a factor (1 + d), |d| <= 2 e, move the
  output by at most 2 e A;
- exp2 and the sums of n terms in fp32: (n + 2^4) 2^-24 (A + |o|);
- bf16 only: each probability is rounded (2^-8 relative, in numerator and
  denominator alike): 2^-8 A; the output is rounded: 2^-8 |o|.
"""
import numpy as np
import pytest
import torch

from gpu_common import require_gpu, say
from paper_2609_01068_amd import binding as B

pytestmark = pytest.mark.gpu
PAGE = 16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


def tables(num_pages, max_slots, max_seq_len):
    from paper_2609_01068_amd.paged import PageTables
    return PageTables(num_pages, max_slots, max_seq_len)


def snapshot(pt):
    return [t.cpu().numpy().copy() for t in (pt.free_bits, pt.page_table, pt.seq_len)]


def free_pages(pt):
    bits = pt.free_bits.cpu().numpy().view(np.uint32)
    return {32 * i + b for i, w in enumerate(bits) for b in range(32) if w >> b & 1}


def check_rows(pt, rows, slots, new, before, n_rows):
    """The layout of an accepted call against its definition."""
    table = pt.page_table.cpu().numpy()
    cu, sm, pos, rs = [], [], [], []
    for s, t in zip(slots, new):
        cu.append(len(pos))
        for j in range(t if s >= 0 else 0):
            p = before[s] + j
            pos.append(p)
            rs.append(s)
            sm.append(table[s, p // PAGE] * PAGE + p % PAGE)
    T = len(pos)
    pad = [-1] * (n_rows - T)
    assert rows.cu.tolist() == cu + [T]
    assert rows.positions.tolist() == pos + pad
    assert rows.row_slot.tolist() == rs + pad
    assert rows.slot_map.tolist() == sm + pad
    return T


@pytest.mark.parametrize("num_pages,slots,max_len,most", [(7, 3, 40, 9), (100, 12, 130, 60), (1000, 70, 700, 300),
                                                          (9000, 600, 3000, 40), (40000, 40, 20000, 4000)])
def test_tables_match_the_host_allocator(num_pages, slots, max_len, most):
    """Prompts, steps and releases in random order, padded batches among them."""
    r = np.random.default_rng(num_pages)
    pt, host = tables(num_pages, slots, max_len), B.Pager(num_pages, PAGE, slots, max_len)
    length = np.zeros(slots, dtype=np.int64)
    for step in range(30):
        busy = np.flatnonzero(length > 0)
        idle = np.flatnonzero(length == 0)
        if len(busy) and r.random() < 0.25:
            gone = r.permutation(busy)[:r.integers(1, len(busy) + 1)]
            assert host.release(gone) == 0
            padded = np.insert(gone, r.integers(0, len(gone) + 1), -1)
            assert pt.release(i32(padded)).item() == 0
            length[gone] = 0
        else:
            kind = "prompt" if len(idle) and (not len(busy) or r.random() < 0.4) else "step"
            ids = r.permutation(idle if kind == "prompt" else busy)
            ids = ids[:r.integers(1, len(ids) + 1)]
            new = r.integers(1, min(most, max_len) + 1, size=len(ids)) if kind == "prompt" else np.ones(len(ids), int)
            rc = host.prefill(ids, new) if kind == "prompt" else host.step(ids)
            n_rows = int(new.sum()) + int(r.integers(0, 5))
            where = r.integers(0, len(ids) + 1)
            slots_in, new_in = np.insert(ids, where, -1), np.insert(new, where, 7)
            was = snapshot(pt)
            rows = pt.append(i32(slots_in), i32(new_in), n_rows)
            st = rows.status.tolist()
            assert st[0] == rc, (step, kind)
            if rc == 0:
                T = check_rows(pt, rows, slots_in, new_in, length, n_rows)
                length[ids] += new
                assert st[1] == T == new.sum()
            else:
                assert all(np.array_equal(a, b) for a, b in zip(was, snapshot(pt)))
                assert st[1:3] == [0, 0] and set(rows.slot_map.tolist()) <= {-1}
            assert st[3] == len(free_pages(pt))
        table = np.array(host.read(B.OUTLETS_META_PAGE_TABLE)).reshape(slots, -1)
        assert np.array_equal(pt.page_table.cpu().numpy(), table), step
        assert pt.seq_len.tolist() == host.read(B.OUTLETS_META_SEQ_LEN) == length.tolist()
        assert free_pages(pt) == set(range(num_pages)) - set(table[table >= 0].tolist())
    host.close()


@pytest.mark.parametrize("n,n_rows", [(1024, 4096), (1025, 4096), (1024, 4097), (3000, 70000)])
def test_large_batches(n, n_rows):
    """Around the sizes where a call's lists leave LDS; many tokens at once
    onto partly filled slots, some of them none."""
    r = np.random.default_rng(n + n_rows)
    pt = tables(2 * n + n_rows // PAGE + 5, n + 3, 400)
    ids = r.permutation(n + 3)[:n]
    length = np.zeros(n + 3, dtype=np.int64)
    for turn in range(3):
        new = r.integers(0, 2 * n_rows // (3 * n), size=n)
        rows = pt.append(i32(ids), i32(new), n_rows)
        assert rows.status[0].item() == 0
        check_rows(pt, rows, ids, new, length, n_rows)
        length[ids] += new
        held = pt.page_table.cpu().numpy()
        used = held[held >= 0]
        assert len(set(used.tolist())) == len(used) == sum(-(-x // PAGE) for x in length)
        assert used.max() == len(used) - 1                  # lowest first
    assert pt.release(i32(ids)).item() == 0
    assert len(free_pages(pt)) == pt.num_pages and pt.page_table.max().item() == -1


@pytest.mark.parametrize("slots,new,n_rows,rc", [
    ([0, 4], [1, 1], 9, B.OUTLETS_ERR_INVALID_ARG),          # no such slot
    ([0, -2], [1, 1], 9, B.OUTLETS_ERR_INVALID_ARG),
    ([1, 3, 1], [1, 1, 1], 9, B.OUTLETS_ERR_INVALID_ARG),    # twice
    ([0, 1], [1, -1], 9, B.OUTLETS_ERR_INVALID_ARG),
    ([0, 1], [1, 71], 200, B.OUTLETS_ERR_INVALID_ARG),       # 30 + 71 > 100
    ([1], [2**31 - 1], 200, B.OUTLETS_ERR_INVALID_ARG),
    ([0, 2], [5, 5], 9, B.OUTLETS_ERR_INVALID_ARG),          # rows
    ([0, 2, 3], [60, 60, 60], 200, B.OUTLETS_ERR_OUT_OF_PAGES),
])
@pytest.mark.parametrize("rows_more", [0, 5000])
def test_refused_appends_change_nothing(slots, new, n_rows, rc, rows_more):
    if slots != [0, 2]:                                 # (too few rows: more would suffice)
        n_rows += rows_more
    pt = tables(11, 4, 100)
    pt.append(i32([1]), i32([30]), 30)
    was = snapshot(pt)
    rows = pt.append(i32(slots), i32(new), n_rows)
    assert rows.status.tolist() == [rc, 0, 0, 9]
    assert rows.cu.tolist() == [0] * (len(slots) + 1)
    for t in (rows.slot_map, rows.positions, rows.row_slot):
        assert t.unique().tolist() == [-1]
    assert all(np.array_equal(a, b) for a, b in zip(was, snapshot(pt)))
    if len(set(slots)) < len(slots) or min(slots) < -1 or max(slots) > 3:
        assert pt.release(i32(slots)).item() == B.OUTLETS_ERR_INVALID_ARG
        assert all(np.array_equal(a, b) for a, b in zip(was, snapshot(pt)))
    rows = pt.append(i32([1, -1, 0]), i32([2, 9, 100]), 200)
    assert rows.status.tolist() == [0, 102, 7, 2]


def test_every_page_and_no_request():
    pt = tables(33, 5, 33 * PAGE)
    rows = pt.append(i32([]), i32([]), 3)
    assert rows.status.tolist() == [0, 0, 0, 33] and rows.cu.tolist() == [0] and rows.slot_map.tolist() == [-1] * 3
    assert pt.append(i32([-1]), i32([4]), 0).status.tolist() == [0, 0, 0, 33]
    assert pt.append(i32([2]), i32([33 * PAGE]), 33 * PAGE).status.tolist() == [0, 33 * PAGE, 33, 0]
    assert pt.page_table[2].tolist() == list(range(33))
    assert pt.append(i32([0]), i32([1]), 1).status.tolist() == [B.OUTLETS_ERR_OUT_OF_PAGES, 0, 0, 0]
    assert pt.release(i32([-1, 0])).item() == 0 and pt.release(i32([2])).item() == 0
    assert len(free_pages(pt)) == 33
    pt.append(i32([1]), i32([20]), 20)
    pt.reset()
    assert len(free_pages(pt)) == 33 and pt.seq_len.tolist() == [0] * 5 and pt.page_table.max().item() == -1


def test_pools_larger_than_the_kept_words():
    """More pages than a call holds words of, with holes that leave few free
    pages here and there."""
    num = 300001
    pt = tables(num, 4, num * PAGE)
    assert pt.append(i32([0]), i32([1 << 20]), 1 << 20).status.tolist() == [0, 1 << 20, 65536, num - 65536]
    for _ in range(3):
        assert pt.append(i32([1]), i32([1 << 20]), 1 << 20).status[0].item() == 0
    assert pt.append(i32([2]), i32([5000]), 5000).status[0].item() == 0
    r = np.random.default_rng(0)
    bits = r.integers(0, 2**32, size=-(-num // 32), dtype=np.uint64).astype(np.uint32) & \
        r.integers(0, 2**32, size=-(-num // 32), dtype=np.uint64).astype(np.uint32)
    bits[:100] = 0
    bits[-1] &= (1 << (num % 32)) - 1
    pt.free_bits.copy_(torch.as_tensor(bits.view(np.int32)))
    free = sorted(free_pages(pt))
    rows = pt.append(i32([3, 2]), i32([900000, 9]), 1 << 20)
    n = 900000 // PAGE + (1 if (5000 + 9 + 15) // PAGE > (5000 + 15) // PAGE else 0)
    assert rows.status.tolist() == [0, 900009, n, len(free) - n]
    assert pt.page_table[3, :900000 // PAGE].tolist() == free[:900000 // PAGE]
    assert sorted(free_pages(pt)) == free[n:]


def test_most_slots():
    """The largest slot count, at both ends of its range."""
    n = 1 << 17
    pt = tables(40, n, 32)
    rows = pt.append(i32([n - 1, 0, n - 2]), i32([17, 3, 32]), 60)
    assert rows.status.tolist() == [0, 52, 5, 35]
    check_rows(pt, rows, [n - 1, 0, n - 2], [17, 3, 32], np.zeros(n, dtype=int), 60)
    assert pt.append(i32([0, n - 1, 0]), i32([1, 1, 1]), 60).status[0].item() == B.OUTLETS_ERR_INVALID_ARG
    assert pt.release(i32([n - 1, n])).item() == B.OUTLETS_ERR_INVALID_ARG
    assert pt.append(i32([-1] * 5000 + [n - 1]), i32([1] * 5001), 5000).status.tolist() == [0, 1, 0, 35]
    assert pt.release(i32([n - 1, -1, 0])).item() == 0 and len(free_pages(pt)) == 38


# ---------------------------------------------------------------- cache write

def make_kv(pt, n_kv, hd, fmt, seed=0, scale=1.0):
    """A cache whose pools hold NaN."""
    from paper_2609_01068_amd.paged import PagedKV
    kv = PagedKV(pt, n_kv, hd, fmt)
    for t in (kv.k_pool, kv.v_pool, kv.block_keys):
        t.fill_(float("nan"))
    return kv


def randn(shape, fmt, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[fmt])


def same_bits(a, b):
    v = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.view(v), b.view(v))


def plain_write(ref, slot_map, k, v):
    kp, vp, bk = ref
    for r, s in enumerate(slot_map):
        if not 0 <= s < len(kp) * PAGE:
            continue
        kp[s // PAGE, :, s % PAGE] = k[r]
        vp[s // PAGE, :, :, s % PAGE] = v[r]
        if s % PAGE == PAGE - 1:
            # in position order: 3e38 + x - 3e38 is 0 in 64 bits for |x| < 2^-54 3e38,
            # whichever x, so with such keys only one order gives the kernel's sum
            total = kp[s // PAGE, :, 0].double()
            for j in range(1, PAGE):
                total = total + kp[s // PAGE, :, j].double()
            bk[s // PAGE] = (total / PAGE).float().to(bk.dtype)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv,layout", [(1, "packed"), (2, "qkv"), (3, "odd"), (8, "qkv")])
def test_cache_write(fmt, hd, n_kv, layout):
    """Prompts that start and end inside pages, then steps that fill pages
    begun by earlier calls; entries outside the pool write nothing.  Copies
    and the 64-bit means are exact."""
    pt = tables(70, 6, 400)
    kv = make_kv(pt, n_kv, hd, fmt)
    ref = [t.clone() for t in (kv.k_pool, kv.v_pool, kv.block_keys)]

    def rows_of(n, seed):
        if layout == "packed":
            return randn((n, n_kv, hd), fmt, seed), randn((n, n_kv, hd), fmt, seed + 1)
        wide = randn((n, (4 + 2 * n_kv) * hd + (1 if layout == "odd" else 0)), fmt, seed)
        at = 4 * hd + (1 if layout == "odd" else 0)
        return wide[:, at:at + n_kv * hd].view(n, n_kv, hd), wide[:, at + n_kv * hd:at + 2 * n_kv * hd].view(n, n_kv, hd)

    calls = [([0, 3, 5], [1, 33, 100]), ([1, 0, 3], [16, 15, 47]), ([0, 1, 3, 5], [1, 1, 1, 1]), ([2, -1], [15, 0]),
             ([2, 5, 0], [1, 11, 14]), ([5, 0], [1, 2])]
    for i, (slots, new) in enumerate(calls):
        T = sum(t for s, t in zip(slots, new) if s >= 0)
        rows = pt.append(i32(slots), i32(new), T + 2)
        assert rows.status[0].item() == 0
        k, v = rows_of(T + 2, 10 * i)
        sm = rows.slot_map.clone()
        if i == 3:
            sm[T] = 70 * PAGE               # behind the pool
            sm[T + 1] = -5
        kv.write(sm, k, v)
        plain_write(ref, sm.tolist(), k, v)
        for a, b, name in zip((kv.k_pool, kv.v_pool, kv.block_keys), ref, ("k", "v", "keys")):
            assert same_bits(a, b), (i, name)


@pytest.mark.parametrize("fmt,hd,T", [("bf16", 128, 2047), ("bf16", 128, 2048), ("f32", 64, 2048), ("bf16", 128, 8192),
                                      ("bf16", 64, 9001), ("f32", 128, 9001), ("bf16", 128, 8191)])
def test_cache_write_of_many_rows(fmt, hd, T):
    """Around the size where tiles grow: prompts behind partly filled pages."""
    n_kv, lens = 3, [1, 17, 900, 2900 if T > 4000 else 333, 40]
    lens.append(T - sum(lens))
    pt = tables(700, 6, 9100)
    kv = make_kv(pt, n_kv, hd, fmt)
    first = pt.append(i32(range(6)), i32([3, 0, 15, 16, 1, 30]), 65)
    k0, v0 = randn((65, n_kv, hd), fmt, 1), randn((65, n_kv, hd), fmt, 2)
    kv.write(first.slot_map, k0, v0)
    rows = pt.append(i32([4, 1, 0, 5, 2, 3]), i32(lens), T)
    assert rows.status[0].item() == 0
    kp, vp, bk = (t.clone() for t in (kv.k_pool, kv.v_pool, kv.block_keys))
    k, v = randn((T, n_kv, hd), fmt, 3), randn((T, n_kv, hd), fmt, 4)
    kv.write(rows.slot_map, k, v)
    at = rows.slot_map.long()
    kp[at // PAGE, :, at % PAGE], vp[at // PAGE, :, :, at % PAGE] = k, v
    full = at[at % PAGE == PAGE - 1] // PAGE
    total = torch.zeros((len(full), n_kv, hd), dtype=torch.float64, device="cuda")
    for j in range(PAGE):
        total = total + kp[full, :, j].double()
    bk[full] = (total / PAGE).float().to(bk.dtype)
    for a, b in zip((kv.k_pool, kv.v_pool, kv.block_keys), (kp, vp, bk)):
        assert same_bits(a, b)


def test_cache_write_without_block_keys_and_scattered():
    """Rows in no page order (each a run of its own), and a cache that holds no block keys."""
    from paper_2609_01068_amd.paged import PagedKV
    pt = tables(20, 2, 320)
    r = np.random.default_rng(0)
    sm = r.permutation(20 * PAGE)[:200]
    sm = sm[sm % PAGE != PAGE - 1]
    pools = dict(k_pool=torch.zeros((20, 2, PAGE, 64), device="cuda"), v_pool=torch.zeros((20, 2, 64, PAGE), device="cuda"))
    kv = PagedKV(pt, 2, 64, "f32", buffers=pools)
    ref = [t.clone() for t in pools.values()] + [torch.zeros((20, 2, 64), device="cuda")]
    k, v = randn((len(sm), 2, 64), "f32", 1), randn((len(sm), 2, 64), "f32", 2)
    kv.write(i32(sm), k, v)
    plain_write(ref, sm.tolist(), k, v)
    assert torch.equal(kv.k_pool, ref[0]) and torch.equal(kv.v_pool, ref[1])
    with pytest.raises(B.OutletsError) as e:
        kv.select(k, i32([0] * len(sm)), i32([0] * len(sm)), 4, 0, 1)
    assert e.value.rc == B.OUTLETS_ERR_INVALID_ARG


def test_block_keys_of_large_and_special_values():
    """Sums in 64 bits: large keys that cancel, infinities, NaN."""
    pt = tables(4, 1, 64)
    for fmt in ("f32", "bf16"):
        kv = make_kv(pt, 1, 64, fmt)
        ref = [t.clone() for t in (kv.k_pool, kv.v_pool, kv.block_keys)]
        k = randn((32, 1, 64), fmt, 5)
        k[0, 0, 0], k[9, 0, 0] = 3e38, -3e38
        k[1:5, 0, 1] = 3e38
        k[3, 0, 2], k[4, 0, 3], k[5, 0, 3], k[6, 0, 4] = float("inf"), float("inf"), float("-inf"), float("nan")
        kv.write(torch.arange(32, dtype=torch.int32, device="cuda"), k, k)
        plain_write(ref, list(range(32)), k, k)
        a, b = kv.block_keys.double(), ref[2].double()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


# ---------------------------------------------------------------- selection

def plain_select(key, q, table, row_slot, pos, n_kv, top_k, sink, local):
    """Index lists by the definition, in numpy float64."""
    n, n_q = q.shape[:2]
    out = np.full((n, n_kv, top_k), -1, dtype=np.int32)
    for r in range(n):
        if row_slot[r] < 0 or pos[r] < 0 or row_slot[r] >= len(table) or pos[r] // PAGE >= table.shape[1]:
            continue
        nb = pos[r] // PAGE + 1
        for g in range(n_kv):
            if nb <= top_k:
                out[r, g, :nb] = np.arange(nb)
                continue
            mid = np.arange(sink, nb - local)
            page = table[row_slot[r], mid]
            s = key[np.clip(page, 0, len(key) - 1), g] @ q[r, g * (n_q // n_kv):(g + 1) * (n_q // n_kv)].T
            s = np.where(np.isnan(s), -np.inf, s).max(axis=1)
            s[(page < 0) | (page >= len(key))] = -np.inf
            best = mid[np.argsort(-s, kind="stable")[:top_k - sink - local]]
            out[r, g] = np.sort(np.concatenate([np.arange(sink), best, np.arange(nb - local, nb)]))
    return out


def scattered(lens, num_pages, max_pages, seed):
    r = np.random.default_rng(seed)
    table = np.full((len(lens) + 1, max_pages), -1, dtype=np.int32)
    ids, at = r.permutation(num_pages), 0
    slots = r.permutation(len(lens) + 1)[:len(lens)]
    for s, n in zip(slots, lens):
        m = -(-n // PAGE)
        table[s, :m] = ids[at:at + m]
        at += m
    return table, slots


def cache_over(table, num_pages, n_kv, hd, fmt, **buffers):
    from paper_2609_01068_amd.paged import PagedKV, PageTables
    pt = PageTables(num_pages, table.shape[0], table.shape[1] * PAGE, buffers=dict(page_table=i32(table)))
    return PagedKV(pt, n_kv, hd, fmt, buffers=buffers)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("hd,n_kv,G", [(64, 2, 2), (128, 8, 4), (128, 1, 1), (64, 3, 5), (128, 2, 8), (128, 2, 16)])
@pytest.mark.parametrize("top_k,sink,local", [(1, 0, 1), (8, 1, 2), (8, 3, 5), (33, 0, 4), (64, 1, 4)])
def test_select(fmt, hd, n_kv, G, top_k, sink, local):
    """Lengths around one page, around top_k pages and long; every page of a row's request at least once."""
    edge = top_k * PAGE
    lens = [1, 16, 17, edge - 1, edge, edge + 1, edge + 17, 2 * edge + 5, 2500, 4803]
    num = sum(-(-n // PAGE) for n in lens) + 5
    table, slots = scattered(lens, num, max(-(-n // PAGE) for n in lens) + 1, top_k)
    keys = randn((num, n_kv, hd), fmt, 3, 0.3)
    kv = cache_over(table, num, n_kv, hd, fmt, block_keys=keys)
    row_slot = np.concatenate([slots, slots[-2:], [-1, slots[0], slots[0], len(table)]]).astype(np.int32)
    pos = np.concatenate([np.array(lens) - 1, [1000, 777], [5, -1, table.shape[1] * PAGE, 3]]).astype(np.int32)
    q = randn((len(pos), n_kv * G, hd), fmt, 4)
    got = kv.select(q, i32(row_slot), i32(pos), top_k, sink, local).cpu().numpy()
    want = plain_select(keys.double().cpu().numpy(), q.double().cpu().numpy(), table, row_slot, pos, n_kv, top_k, sink,
                        local)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_select_ties_and_special_keys(fmt):
    """Equal scores go to the lowest page; +-inf and NaN keys; keys of pages
    that are not visible are not looked at; q rows apart and odd."""
    n_kv, G, hd, top_k = 2, 3, 128, 12
    table, slots = scattered([2000, 2000, 2000, 2000], 520, 126, 1)
    keys = randn((520, n_kv, hd), fmt, 3, 0.3)
    k = keys.clone()
    p0, p1, p2, p3 = (table[s] for s in slots)
    k[p0[:125]] = k[p0[0]].clone()                             # all equal
    k[p1[20:60]] = k[p1[20]].clone()                           # forty equal ones
    k[p2[30], 0, 5], k[p2[31], 0, 6], k[p2[32], 1, :] = float("nan"), float("inf"), float("nan")
    k[p2[40], :, 7] = float("-inf")
    k[p3[100:125]] = float("nan")                              # behind the positions used below
    spare = sorted(set(range(520)) - set(table.reshape(-1).tolist()))
    k[spare] = float("nan")
    kv = cache_over(table, 520, n_kv, hd, fmt, block_keys=k)
    row_slot = np.array([slots[0], slots[1], slots[2], slots[2], slots[3], slots[3]], dtype=np.int32)
    pos = np.array([1999, 1999, 1999, 1500, 1599, 200], dtype=np.int32)
    wide = randn((6, n_kv * G * hd + 3), fmt, 9)
    wide[0] = 0                                                # every score 0, some of them -0
    q = wide[:, 3:].view(6, n_kv * G, hd)
    got = kv.select(q, i32(row_slot), i32(pos), top_k, 1, 2).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = plain_select(k.double().cpu().numpy(), q.double().cpu().numpy(), table, row_slot, pos, n_kv, top_k, 1, 2)
    assert np.array_equal(got, want)
    assert got[0, 0].tolist() == list(range(10)) + [123, 124]


def test_select_in_parts(monkeypatch):
    """A workspace of a few rows: the same selection, part by part; tables with holes."""
    from paper_2609_01068_amd import paged
    table, slots = scattered([3000] * 7, 1400, 190, 2)
    table[slots[0], 50:60] = -1
    table[slots[1], 70] = 1400
    keys = randn((1400, 2, 64), "bf16", 3)
    kv = cache_over(table, 1400, 2, 64, "bf16", block_keys=keys)
    rs, pos = np.repeat(slots, 3).astype(np.int32), np.arange(2900, 2921, dtype=np.int32)
    q = randn((21, 8, 64), "bf16", 4)
    want = plain_select(keys.double().cpu().numpy(), q.double().cpu().numpy(), table, rs, pos, 2, 20, 1, 2)
    assert np.array_equal(kv.select(q, i32(rs), i32(pos), 20, 1, 2).cpu().numpy(), want)
    for rows in (1, 4):
        monkeypatch.setattr(paged, "_SELECT_WS", rows * 190 * 2 * 8 + 100)
        assert np.array_equal(kv.select(q, i32(rs), i32(pos), 20, 1, 2).cpu().numpy(), want)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["ties", "near", "overflow", "nan", "zero", "holes"])
def test_select_crowded_borders(fmt, kind):
    """More pages near the border than are compared one with another: equal
    scores, scores that only 64 bits tell apart, products past the fp32
    range, NaN, and zero queries."""
    n_kv, G, hd, top_k = 2, 4, 128, 40
    table, slots = scattered([16 * 700, 16 * 430 + 3, 16 * 50], 1200, 710, 4)
    k = randn((1200, n_kv, hd), fmt, 3, 0.3)
    q = randn((3, n_kv * G, hd), fmt, 4)
    if kind in ("ties", "near"):
        k[:] = k[0].clone()
        if kind == "near":                          # 2^-30 apart, and in no page order
            k[:, :, 17] = (2.0**-30 * torch.randperm(1200, device="cuda").add(1)[:, None] / 4096).to(k.dtype)
            q[:, :, 17] = 1.0
        else:
            k[torch.as_tensor(table[slots[0], [5, 300, 650]].astype(np.int64), device="cuda")] *= 1.5
    elif kind == "overflow":
        k[:, :, 3] = 3e38 * torch.sign(k[:, :, 3])
        q[:, :, 3] = 8.0
    elif kind == "nan":
        k[torch.as_tensor(table[slots[0], 100].astype(np.int64), device="cuda")] = float("nan")
        q[1, 3, 7] = float("nan")
        q[2] = float("inf")
    elif kind == "zero":
        q[0] = 0
        k[:, :, 9] = -0.0
    else:
        table[slots[0], 20:690] = -1
        table[slots[1], 2:400:2] = 1200
    kv = cache_over(table, 1200, n_kv, hd, fmt, block_keys=k)
    pos = np.array([16 * 700 - 1, 16 * 430 + 2, 16 * 50 - 1], dtype=np.int32)
    got = kv.select(q, i32(slots), i32(pos), top_k, 2, 3).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = plain_select(k.double().cpu().numpy(), q.double().cpu().numpy(), table, slots, pos, n_kv, top_k, 2, 3)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt,G", [("f32", 2), ("bf16", 1), ("bf16", 2), ("bf16", 4), ("bf16", 8), ("bf16", 16)])
@pytest.mark.parametrize("lens", [(4000, 4000), (170000,), (210000, 9000)])
def test_select_long_and_shared(fmt, G, lens):
    """Consecutive rows of one request beside rows of another, in tables whose
    scores fit LDS for several rows, for none while chunks are scored apart,
    and not at all."""
    n_kv, hd, top_k = 2, 64, 48
    num = sum(-(-n // PAGE) for n in lens) + 3
    table, slots = scattered(lens, num, max(-(-n // PAGE) for n in lens), 4)
    k = randn((num, n_kv, hd), fmt, 3, 0.3)
    kv = cache_over(table, num, n_kv, hd, fmt, block_keys=k)
    row_slot, pos = [], []
    for s, n in zip(slots, lens):
        for t in (5, 18):
            row_slot += [s] * t + [-1]
            pos += list(range(n - t, n)) + [0]
    pos[3], pos[6] = 100, lens[0] // 2
    q = randn((len(pos), n_kv * G, hd), fmt, 4)
    got = kv.select(q, i32(row_slot), i32(pos), top_k, 1, 2).cpu().numpy()
    want = plain_select(k.double().cpu().numpy(), q.double().cpu().numpy(), table, row_slot, pos, n_kv, top_k, 1, 2)
    assert np.array_equal(got, want)


# ---------------------------------------------------------------- attention

@pytest.mark.parametrize("fmt,G", [("f32", 2), ("bf16", 1), ("bf16", 4), ("bf16", 16)])
@pytest.mark.parametrize("parts", [1, 3])
def test_select_short_rows_of_long_tables(monkeypatch, fmt, G, parts):
    """Tables of more than 1,024 pages, and rows of fewer, of as many and of
    more; alone, side by side with a row of the same slot, and with none to see."""
    from paper_2609_01068_amd import paged
    n_kv, hd, n, slots, width, top_k = 8, 64, 171, 128, 1300, 24
    r = np.random.default_rng(G)
    table = r.integers(0, 2000, size=(slots, width)).astype(np.int32)
    pages = r.choice([1, 24, 25, 90, 300, 1023, 1024, 1025, 1300], size=n)
    rs = r.integers(0, slots, size=n).astype(np.int32)
    rs[16:48], rs[64:71], rs[-3:] = 5, 7, 9
    pages[32:48] = np.minimum(pages[32:48], 1024)
    pos = (pages * PAGE - 1 - r.integers(0, PAGE, size=n)).astype(np.int32)
    rs[3], pos[20], rs[50], pos[60] = -1, -1, slots, width * PAGE
    keys, q = randn((2000, n_kv, hd), fmt, 3, 0.3), randn((n, n_kv * G, hd), fmt, 4)
    kv = cache_over(table, 2000, n_kv, hd, fmt, block_keys=keys)
    if parts > 1:
        monkeypatch.setattr(paged, "_SELECT_WS", n * n_kv * width * 12 // parts)
    want = plain_select(keys.double().cpu().numpy(), q.double().cpu().numpy(), table, rs, pos, n_kv, top_k, 1, 3)
    for _ in range(2):
        assert np.array_equal(kv.select(q, i32(rs), i32(pos), top_k, 1, 3).cpu().numpy(), want)


def attention_ref(kp, vp, q, table, row_slot, pos, sel, gate):
    """Output and error bound (without the rounding of bf16) in numpy float64."""
    n, n_q, hd = q.shape
    n_kv = kp.shape[1]
    G = n_q // n_kv
    out, e32, e16 = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    for r in range(n):
        if row_slot[r] < 0 or pos[r] < 0 or row_slot[r] >= len(table) or pos[r] // PAGE >= table.shape[1]:
            continue
        for g in range(n_kv):
            K, V = [], []
            for b in sel[r, g]:
                if b < 0 or b > pos[r] // PAGE or b >= table.shape[1]:
                    continue
                page = table[row_slot[r], b]
                if not 0 <= page < len(kp):
                    continue
                m = min(PAGE, pos[r] + 1 - b * PAGE)
                K.append(kp[page, g, :m])
                V.append(vp[page, g, :, :m].T)
            if not K:
                continue
            K, V = np.concatenate(K), np.concatenate(V)
            h = slice(g * G, (g + 1) * G)
            s = q[r, h] @ K.T / np.sqrt(hd)
            w = np.exp(s - s.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            o = w @ V
            A = np.einsum("hk,hkc->hc", w, np.abs(V[None] - o[:, None]))
            e = ((hd + 2) * 2.0**-24 * (np.abs(q[r, h]) @ np.abs(K).T) / np.sqrt(hd)).max(axis=1, keepdims=True)
            out[r, h] = o
            e32[r, h] = 2 * e * A + (len(K) + 16) * 2.0**-24 * (A + np.abs(o))
            e16[r, h] = 2.0**-8 * A
    if gate is not None:
        f = 1 / (1 + np.exp(-gate))
        out, e32, e16 = out * f, e32 * f + 2.0**-20 * np.abs(out * f), e16 * f
    return out, e32, e16


def check_attention(kv, q, table, row_slot, pos, sel, gate=None, out=None):
    got = kv.attend(q, i32(row_slot), i32(pos), i32(sel), gate=gate, out=out)
    f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    ref, e32, e16 = attention_ref(f(kv.k_pool), f(kv.v_pool), f(q), table, row_slot, pos, sel, f(gate))
    # 1.01: products of the first-order bounds
    tol = 1.01 * (e32 + (e16 + 2.0**-8 * np.abs(ref) if kv.fmt == "bf16" else 2.0**-24 * np.abs(ref)))
    d = np.abs(f(got) - ref)
    assert np.isfinite(d).all() and (d <= tol).all(), (d - tol).max()
    return got


def random_sel(pos, n_kv, top_k, seed):
    """Distinct visible pages in random order, some entries -1."""
    r = np.random.default_rng(seed)
    sel = np.full((len(pos), n_kv, top_k), -1, dtype=np.int32)
    for i, p in enumerate(pos):
        for g in range(n_kv):
            nb = max(p, 0) // PAGE + 1
            pick = r.permutation(nb)[:r.integers(1, top_k + 1)]
            if i % 2:
                pick[0] = nb - 1 if nb - 1 not in pick else pick[0]
            sel[i, g, r.permutation(top_k)[:len(pick)]] = pick
    return sel


def fill_pages(table, lens, slots, num, n_kv, hd, fmt, scale=1.0):
    """Pools that hold NaN wherever no token of a request stands."""
    k, v = (torch.full(s, float("nan"), dtype=DT[fmt], device="cuda") for s in
            ((num, n_kv, PAGE, hd), (num, n_kv, hd, PAGE)))
    for i, (s, n) in enumerate(zip(slots, lens)):
        pages = torch.as_tensor(table[s, :-(-n // PAGE)].astype(np.int64), device="cuda")
        a, b = (randn((len(pages), n_kv, PAGE, hd), fmt, 100 + 2 * i + j, scale if j == 0 else 1.0) for j in (0, 1))
        if n % PAGE:
            a[-1, :, n % PAGE:] = float("nan")
            b[-1, :, n % PAGE:] = float("nan")
        k[pages], v[pages] = a, b.transpose(2, 3)
    return k, v


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("hd,n_kv,G", [(64, 2, 2), (128, 8, 4), (128, 1, 1), (64, 3, 5), (128, 2, 8), (128, 2, 16)])
@pytest.mark.parametrize("top_k", [1, 3, 8, 64, 130])
def test_attention(fmt, hd, n_kv, G, top_k):
    lens = [1, 2, 15, 16, 17, 33, 500, 2100]
    num = sum(-(-n // PAGE) for n in lens) + 3
    table, slots = scattered(lens, num, 133, 7)
    k, v = fill_pages(table, lens, slots, num, n_kv, hd, fmt)
    kv = cache_over(table, num, n_kv, hd, fmt, k_pool=k, v_pool=v)
    row_slot = np.concatenate([slots, [slots[-1], slots[-2]]]).astype(np.int32)
    pos = np.concatenate([np.array(lens) - 1, [999, 495]]).astype(np.int32)
    wide = randn((len(pos), 3 * n_kv * G * hd), fmt, 5)
    q = wide[:, :n_kv * G * hd].view(len(pos), n_kv * G, hd)
    gate = wide[:, -n_kv * G * hd:].view(len(pos), n_kv * G, hd) if top_k % 2 else None
    sel = random_sel(pos, n_kv, top_k, top_k)
    check_attention(kv, q, table, row_slot, pos, sel, gate)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_attention_edges(fmt):
    """Rows without keys, bad entries, entries twice, bad table pages, an
    output inside a wider buffer; padding rows are zeros and what lies between
    the output's rows stays."""
    lens, n_kv, G, hd = [300, 300, 40], 2, 4, 64
    table, slots = scattered(lens, 60, 20, 3)
    k, v = fill_pages(table, lens, slots, 60, n_kv, hd, fmt, 4.0)
    broken = table.copy()
    broken[slots[1], 3], broken[slots[1], 4] = -1, 60
    kv = cache_over(broken, 60, n_kv, hd, fmt, k_pool=k, v_pool=v)
    row_slot = np.array([slots[0], -1, slots[1], slots[0], slots[2], len(table), slots[0], slots[1]], dtype=np.int32)
    pos = np.array([299, 20, 299, -1, 39, 20, 130, 299], dtype=np.int32)
    sel = np.full((8, n_kv, 6), -1, dtype=np.int32)
    sel[0, 0] = [0, 0, 18, 18, 5, 0]                # twice, three times
    sel[0, 1] = [-1, -7, 19, 2**31 - 1, -2**31, -1]     # none of the row's
    sel[1] = [0, 1, 2, 3, 4, 5]
    sel[2] = [3, 4, -1, 9, 4, 3]                    # 3 and 4 are no pages
    sel[3] = [0, 1, 2, 3, 4, 5]
    sel[4, 0], sel[4, 1] = [2, 1, 0, -1, -1, -1], [1, 3, 4, 5, 6, 7]
    sel[5] = 0
    sel[6] = [8, 9, 10, 1, 18, 0]                   # 9 and up are behind the position
    sel[7] = [3, 4, 3, 4, -1, -1]
    wide = torch.full((8, n_kv * G * hd + 16), 7.0, dtype=DT[fmt], device="cuda")
    out = wide[:, :n_kv * G * hd].view(8, n_kv * G, hd)
    q = randn((8, n_kv * G, hd), fmt, 5)
    got = check_attention(kv, q, broken, row_slot, pos, sel, out=out)
    assert got.data_ptr() == wide.data_ptr() and (wide[:, n_kv * G * hd:] == 7.0).all()
    for r in (1, 3, 5, 7):
        assert (got[r] == 0).all()
    assert (got[0, G:] == 0).all() and (got[0, :G] != 0).any()


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_attention_of_large_scores_and_infinities(fmt):
    """Scores far apart in any order (the running maximum moves); an infinite
    key far below every other weighs nothing; a NaN key of a read page shows."""
    n_kv, G, hd = 1, 2, 128
    table, slots = scattered([640], 41, 40, 3)
    k, v = fill_pages(table, [640], slots, 41, n_kv, hd, fmt, 8.0)
    q = randn((1, 2, hd), fmt, 5, 3.0)
    kv = cache_over(table, 41, n_kv, hd, fmt, k_pool=k, v_pool=v)
    sel = np.random.default_rng(0).permutation(40).astype(np.int32).reshape(1, 1, 40)
    got = check_attention(kv, q, table, slots[:1].astype(np.int32), np.array([639]), sel)
    q[:, :, 0] = 1.0
    page = table[slots[0], 7]
    k[page, 0, 3, 0] = float("-inf")
    one = kv.attend(q, i32(slots[:1]), i32([639]), i32(sel))
    assert one.isfinite().all()
    k[page, 0, 3, 0] = float("nan")
    assert kv.attend(q, i32(slots[:1]), i32([639]), i32(sel)).isnan().all()
    assert got.isfinite().all()


@pytest.mark.parametrize("rows", [1, 2, 37, 700])
def test_attention_row_counts(rows):
    """Few rows over many pages and many rows, on one cache."""
    n_kv, G, hd, top_k = 2, 4, 128, 200
    table, slots = scattered([4000], 260, 250, 5)
    k, v = fill_pages(table, [4000], slots, 260, n_kv, hd, "bf16")
    kv = cache_over(table, 260, n_kv, hd, "bf16", k_pool=k, v_pool=v)
    pos = np.linspace(3999, 10, rows).astype(np.int32)
    sel = random_sel(pos, n_kv, top_k, rows)
    q = randn((rows, n_kv * G, hd), "bf16", 6)
    check_attention(kv, q, table, np.repeat(slots[:1], rows).astype(np.int32), pos, sel)


@pytest.mark.parametrize("hd,G", [(128, 1), (64, 2), (128, 3), (128, 4), (64, 8)])
@pytest.mark.parametrize("kind", ["plain", "nan", "inf", "twice", "mixed"])
def test_attention_of_rows_that_share_a_slot(hd, G, kind):
    """A prompt's rows: pages that only some of them select, whose values are
    infinite or NaN, must not show in the others; a page listed twice by one
    row; a padding row and rows of another slot between them."""
    n_kv, top_k, rows = 2, 24, 600
    lens = [1500, 700]
    table, slots = scattered(lens, 150, 100, 5)
    k, v = fill_pages(table, lens, slots, 150, n_kv, hd, "bf16")
    kv = cache_over(table, 150, n_kv, hd, "bf16", k_pool=k, v_pool=v)
    pos = np.arange(900, 900 + rows, dtype=np.int32)
    row_slot = np.repeat(slots[:1], rows).astype(np.int32)
    sel = np.full((rows, n_kv, top_k), -1, dtype=np.int32)
    r = np.random.default_rng(G)
    for i in range(rows):
        for g in range(n_kv):
            sel[i, g] = np.sort(r.permutation(40)[:top_k])
        if i % 16 == 5:
            sel[i] = -1
        elif i % 3 == 0:
            sel[i, :, -1] = pos[i] // PAGE
    if kind in ("nan", "inf"):
        page = table[slots[0], 17]
        (k if kind == "nan" and G % 2 else v)[page, :, 3, 5] = float(kind)
    elif kind == "twice":
        sel[7, 1, 2] = sel[7, 1, 9]
        sel[100:120, 0, :3] = sel[100:120, 0, 3:4]
    elif kind == "mixed":
        row_slot[10], row_slot[33] = -1, slots[1]
        pos[33], pos[50], pos[70] = 650, -1, 100000
        row_slot[200:203] = len(table)
    q = randn((rows, n_kv * G, hd), "bf16", 6)
    got = kv.attend(q, i32(row_slot), i32(pos), i32(sel)).double().cpu().numpy()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        ref, e32, e16 = attention_ref(f(kv.k_pool), f(kv.v_pool), f(q), table, row_slot, pos, sel, None)
        tol = 1.01 * (e32 + e16 + 2.0**-8 * np.abs(ref))
        bad = ~(np.abs(got - ref) <= tol)
    if kind in ("nan", "inf"):
        hit = (sel == 17).any(axis=2).repeat(G, axis=1)                     # [rows, heads]
        assert hit.any() and not hit.all() and np.isfinite(got[~hit]).all() and not bad[~hit].any()
        assert not np.isfinite(got[hit]).all(axis=1).any()
    else:
        assert not bad.any()


def test_select_of_denormal_and_huge_values():
    """Keys below the normal range under large queries: scores of ordinary
    size, which an instruction that drops denormals would lose."""
    n_kv, G, hd, top_k = 1, 4, 128, 20
    table, slots = scattered([1600], 101, 100, 4)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    step = torch.randint(-100, 101, (101, n_kv, hd), generator=g, device="cuda")
    for fmt, unit, scale in (("bf16", 2.0**-133, 2.0**120), ("f32", 2.0**-149, 2.0**127)):
        k = (step.double() * unit).to(DT[fmt])
        q = randn((1, n_kv * G, hd), fmt, 4) * scale
        kv = cache_over(table, 101, n_kv, hd, fmt, block_keys=k)
        got = kv.select(q, i32(slots), i32([1599]), top_k, 1, 2).cpu().numpy()
        with np.errstate(invalid="ignore"):             # the largest queries are infinite
            want = plain_select(k.double().cpu().numpy(), q.double().cpu().numpy(), table, slots, [1599], n_kv, top_k, 1, 2)
        assert np.array_equal(got, want), fmt


def test_pools_past_32_bit_offsets():
    """Pages whose elements lie behind 2^31: write, select, attend."""
    from paper_2609_01068_amd.paged import PagedKV, PageTables
    n_kv, G, hd, num, top_k = 8, 4, 128, 140000, 9
    pt = PageTables(num, 3, 700)
    pt.free_bits.zero_()
    last = torch.arange(num - 128, num, device="cuda")
    pt.free_bits[-4:] = -1                              # the pool ends on a whole word
    kv = PagedKV(pt, n_kv, hd, "bf16")
    assert kv.k_pool.numel() > 2**31 + 2**27
    rows = pt.append(i32([2, 0, 1]), i32([640, 333, 700]), 1673)
    assert rows.status[0].item() == 0 and pt.page_table[2].min().item() == -1
    k, v = randn((1673, n_kv, hd), "bf16", 1), randn((1673, n_kv, hd), "bf16", 2)
    kv.write(rows.slot_map, k, v)
    at = rows.slot_map.long()
    assert at.min().item() // PAGE >= num - 128
    assert torch.equal(kv.k_pool[at // PAGE, :, at % PAGE], k) and torch.equal(kv.v_pool[at // PAGE, :, :, at % PAGE], v)
    # the same on the last pages alone, renumbered
    table = pt.page_table.cpu().numpy()
    small = np.where(table >= 0, table - (num - 128), -1)
    f = lambda t: t[last].double().cpu().numpy()  # noqa: E731
    rs, pos = np.array([2, 0, 1], dtype=np.int32), np.array([639, 332, 699], dtype=np.int32)
    q = randn((3, n_kv * G, hd), "bf16", 3)
    sel = kv.select(q, i32(rs), i32(pos), top_k, 1, 2)
    want = plain_select(f(kv.block_keys), q.double().cpu().numpy(), small, rs, pos, n_kv, top_k, 1, 2)
    assert np.array_equal(sel.cpu().numpy(), want)
    got = kv.attend(q, i32(rs), i32(pos), sel).double().cpu().numpy()
    ref, e32, e16 = attention_ref(f(kv.k_pool), f(kv.v_pool), q.double().cpu().numpy(), small, rs, pos, want, None)
    assert (np.abs(got - ref) <= 1.01 * (e32 + e16 + 2.0**-8 * np.abs(ref))).all()


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_more_rows_than_one_launch(fmt):
    """Rows past a grid's limit, of slots that change every row and of one slot."""
    n, n_kv, G, hd, top_k, slots = 70001, 1, 2, 64, 2, 7
    table = np.arange(slots * 4, dtype=np.int32).reshape(slots, 4)
    r = np.random.default_rng(0)
    row_slot = np.where(np.arange(n) < 40000, np.arange(n) % slots, 3).astype(np.int32)
    pos = r.integers(0, 64, size=n).astype(np.int32)
    k, v = randn((28, n_kv, PAGE, hd), fmt, 1), randn((28, n_kv, hd, PAGE), fmt, 2)
    keys = (k.double().mean(dim=2)).to(DT[fmt])
    kv = cache_over(table, 28, n_kv, hd, fmt, k_pool=k, v_pool=v, block_keys=keys)
    q = randn((n, n_kv * G, hd), fmt, 3)
    sel = kv.select(q, i32(row_slot), i32(pos), top_k, 0, 1)
    got = kv.attend(q, i32(row_slot), i32(pos), sel)
    rows = np.unique(np.concatenate([r.integers(0, n, size=300), [0, 32767, 32768, 32769, 39999, 40000, 65535, 65536, n - 1]]))
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = plain_select(f(keys), f(q[rows]), table, row_slot[rows], pos[rows], n_kv, top_k, 0, 1)
    assert np.array_equal(sel[rows].cpu().numpy(), want)
    ref, e32, e16 = attention_ref(f(k), f(v), f(q[rows]), table, row_slot[rows], pos[rows], want, None)
    tol = 1.01 * (e32 + (e16 + 2.0**-8 * np.abs(ref) if fmt == "bf16" else 2.0**-24 * np.abs(ref)))
    assert (np.abs(f(got[rows]) - ref) <= tol).all()


# ---------------------------------------------------------------- together

class Serving:
    """A decode loop over the operators, as a serving program runs them."""

    def __init__(self, fmt="bf16", n_kv=2, G=4, hd=128, slots=6, max_len=700, top_k=9, pages=200):
        self.pt = tables(pages, slots, max_len)
        self.kv = make_kv(self.pt, n_kv, hd, fmt)
        self.shape, self.top_k, self.fmt = (n_kv, G, hd), top_k, fmt

    def step(self, slots, new, n_rows, qkv):
        n_kv, G, hd = self.shape
        q, k, v = (t.view(n_rows, -1, hd) for t in qkv.split([n_kv * G * hd, n_kv * hd, n_kv * hd], dim=1))
        rows = self.pt.append(slots, new, n_rows)
        self.kv.write(rows.slot_map, k, v)
        sel = self.kv.select(q, rows.row_slot, rows.positions, self.top_k, 1, 2)
        return rows, sel, self.kv.attend(q, rows.row_slot, rows.positions, sel)

    def check(self, rows, sel, out, qkv):
        n_kv, G, hd = self.shape
        q = qkv[:, :n_kv * G * hd].view(len(out), -1, hd)
        table, rs, pos = self.pt.page_table.cpu().numpy(), rows.row_slot.cpu().numpy(), rows.positions.cpu().numpy()
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        want = plain_select(f(self.kv.block_keys), f(q), table, rs, pos, n_kv, self.top_k, 1, 2)
        assert np.array_equal(sel.cpu().numpy(), want)
        ref, e32, e16 = attention_ref(f(self.kv.k_pool), f(self.kv.v_pool), f(q), table, rs, pos, want, None)
        tol = 1.01 * (e32 + (e16 + 2.0**-8 * np.abs(ref) if self.fmt == "bf16" else 2.0**-24 * np.abs(ref)))
        assert (np.abs(f(out) - ref) <= tol).all()


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_serving_loop(fmt):
    """Prompts, single tokens, several tokens at once, leaving and coming requests."""
    s = Serving(fmt)
    n_kv, G, hd = s.shape
    calls = [([4, 0], [333, 20]), ([0, 4, -1], [1, 1, 0]), ([2, 0, 4], [40, 5, 1]), ([0, 2, 4], [1, 8, 3]), ([1], [600]),
             ([4, 1, 0, 2], [1, 1, 1, 1])]
    for i, (slots, new) in enumerate(calls):
        if i == 4:
            assert s.pt.release(i32([4])).item() == 0
        T = sum(t for a, t in zip(slots, new) if a >= 0)
        qkv = randn((T + 1, (G + 2) * n_kv * hd), fmt, i)
        rows, sel, out = s.step(i32(slots), i32(new), T + 1, qkv)
        assert rows.status[0].item() == 0
        s.check(rows, sel, out, qkv)
        assert (out[T] == 0).all()


def test_captured_step():
    """A step captured once and replayed while the requests grow, with eager
    work between the replays, against the same steps run eagerly; then a
    second graph of the same cache and a step on another stream."""
    live, eager = Serving(), Serving()
    n_kv, G, hd = live.shape
    prompt = randn((400, (G + 2) * n_kv * hd), "bf16", 50)
    for s in (live, eager):
        s.step(i32([0, 3, 5]), i32([300, 13, 87]), 400, prompt)
    slots, new = i32([3, 5, -1, 0]), i32([1, 1, 1, 1])
    qkv = torch.zeros((4, (G + 2) * n_kv * hd), dtype=torch.bfloat16, device="cuda")
    saved = snapshot(live.pt)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                    # warm up on a side stream, then take the step back
        live.step(slots, new, 4, qkv)
    side.synchronize()
    for t, x in zip((live.pt.free_bits, live.pt.page_table, live.pt.seq_len), saved):
        t.copy_(torch.as_tensor(x))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, live.step(slots, new, 4, qkv)))
    torch.cuda.synchronize()
    for i in range(24):
        x = randn(qkv.shape, "bf16", 60 + i)
        qkv.copy_(x)
        graph, (rows, sel, out) = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        r2, s2, o2 = eager.step(slots, new, 4, x)
        for a, b in zip(list(rows) + [sel, out], list(r2) + [s2, o2]):
            assert torch.equal(a, b), i
        live.check(rows, sel, out, x)
        assert sum(torch.ones(1000, device="cuda").sum().item() for _ in range(2)) == 2000
    x = randn(qkv.shape, "bf16", 99)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        rows, sel, out = live.step(slots, new, 4, x)
    side.synchronize()
    live.check(rows, sel, out, x)


def test_stream_argument():
    pt = tables(20, 2, 200)
    side = torch.cuda.Stream()
    a, b = i32([0, 1]), i32([100, 30])
    torch.cuda.synchronize()
    rows = pt.append(a, b, 130, stream=side)
    side.synchronize()
    assert rows.status.tolist() == [0, 130, 9, 11]


def test_wrapper_refusals():
    s = Serving()
    n_kv, G, hd = s.shape
    q = randn((2, n_kv * G, hd), "bf16", 0)
    rs, pos, sel = i32([0, 1]), i32([3, 4]), torch.zeros((2, n_kv, 4), dtype=torch.int32, device="cuda")
    for bad in (lambda: s.pt.append(rs.long(), rs, 4), lambda: s.pt.append(rs, i32([1]), 4), lambda: s.pt.append(rs.cpu(), rs, 4),
                lambda: s.pt.release(rs[::2].float()), lambda: s.kv.write(rs, q, q), lambda: s.kv.write(rs, q[:, :n_kv].float(), q[:, :n_kv]),
                lambda: s.kv.select(q, rs, i32([1]), 4), lambda: s.kv.select(q.float(), rs, pos, 4),
                lambda: s.kv.attend(q, rs, pos, sel[:1]), lambda: s.kv.attend(q, rs, pos, sel.long()),
                lambda: s.kv.attend(q, rs, pos, sel, gate=q[:, :1])):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        s.kv.attend(randn((2, hd, n_kv * G), "bf16", 0).transpose(1, 2), rs, pos, sel)
    with pytest.raises(B.OutletsError) as e:
        s.kv.select(q, rs, pos, 4, 3, 2)
    assert e.value.rc == B.OUTLETS_ERR_INVALID_ARG
    with pytest.raises(B.OutletsError) as e:
        s.kv.attend(randn((2, n_kv * G * hd + 1), "bf16", 0)[:, 1:].view(2, n_kv * G, hd), rs, pos, sel)
    assert e.value.rc == B.OUTLETS_ERR_UNSUPPORTED
    say("wrapper refusals")
