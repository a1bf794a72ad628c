"""Sparse attention in decode steps (outlets_sparse_steps): block keys, the
selection and the attention output of every step against 64-bit forms of the
cache and the queries that the step used; steps of short caches and contexts
with it off keep their bits.  Attention tolerances as in test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from gpu_common import (device_states, make_case, make_predictor, reduced_shape, require_gpu, say,
                        step_inputs, tensor_to_f64)
from paper_2609_01068_amd import binding as B
from test_gpu_paged import PAGE, attention_ref, plain_select, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def read(pred, case):
    """The context's pools, block keys, page table and lengths after a call."""
    m, dt = case.wl.shape, pred.act_dtype
    num = pred.cfg.num_pages
    out = {"K": pred.buffer("K_POOL", dt).view(num, m.n_kv, PAGE, m.head_dim),
           "V": pred.buffer("V_POOL", dt).view(num, m.n_kv, m.head_dim, PAGE),
           "keys": pred.buffer("BLOCK_KEYS", dt).view(num, m.n_kv, m.head_dim)}
    out["table"] = pred.meta(B.OUTLETS_META_PAGE_TABLE).reshape(pred.cfg.max_slots, -1)
    out["len"] = pred.meta(B.OUTLETS_META_SEQ_LEN)
    return out


def check_block_keys(r):
    """Every full page's block key is the 64-bit mean of its keys, in position order."""
    pages = [r["table"][s, i] for s in range(len(r["len"])) for i in range(r["len"][s] // PAGE)]
    at = torch.as_tensor(np.array(pages, dtype=np.int64), device="cuda")
    K = r["K"][at].double()
    total = K[:, :, 0]
    for j in range(1, PAGE):
        total = total + K[:, :, j]
    assert same_bits(r["keys"][at], (total / PAGE).float().to(r["keys"].dtype))


def check_step(pred, case, slots, top_k, sink, local):
    m, r = case.wl.shape, read(pred, case)
    check_block_keys(r)
    n = len(slots)
    q = tensor_to_f64(pred.buffer("Q", pred.act_dtype)).reshape(n, m.n_q, m.head_dim)
    pos = (r["len"][slots] - 1).astype(np.int32)
    if pos.max() // PAGE + 1 <= top_k:               # nothing to select from: the step was not sparse
        with pytest.raises(B.OutletsError):
            pred.buffer("SELECTED", torch.int32)
        return
    want = plain_select(tensor_to_f64(r["keys"]), q, r["table"], slots, pos, m.n_kv, top_k, sink, local)
    sel = pred.buffer("SELECTED", torch.int32).view(n, m.n_kv, top_k).cpu().numpy()
    assert np.array_equal(sel, want)
    got = tensor_to_f64(pred.buffer("ATTN", pred.act_dtype)).reshape(n, m.n_q, m.head_dim)
    ref, e32, e16 = attention_ref(tensor_to_f64(r["K"]), tensor_to_f64(r["V"]), q, r["table"], slots, pos, want, None)
    if case.wl.attn_gate:
        # the gate values are rounded to the activation format (2^-8 relative;
        # the sigmoid's slope is at most 1/4) after a product of d terms
        a = tensor_to_f64(pred.buffer("NORM_ATTN", pred.act_dtype)).reshape(n, -1)
        w = pred.tensors["w_attn_gate"].double().cpu().numpy()
        g = a @ w.T
        slack = (2.0**-8 * np.abs(g) + m.d * 2.0**-24 * (np.abs(a) @ np.abs(w).T)) / 4
        f = (1 / (1 + np.exp(-g))).reshape(ref.shape)
        e32 = e32 * f + np.abs(ref) * slack.reshape(ref.shape)
        ref, e16 = ref * f, e16 * f
    tol = 1.01 * (e32 + (e16 + 2.0**-8 * np.abs(ref) if pred.act_dtype == torch.bfloat16 else 2.0**-24 * np.abs(ref)))
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) - tol).max()


CASES = {
    "tiny fp32": lambda: make_case(0, lens=[300, 16, 190, 97]),
    "bf16": lambda: make_case(1, lens=[500, 17, 1200, 96, 128], shape=reduced_shape(), n_req=5),
    "bf16 gated": lambda: make_case(1, lens=[500, 17, 1200, 96, 128], shape=reduced_shape(), n_req=5, attn_gate=True),
    "e4m3": lambda: make_case(4, lens=[700, 130, 15], shape=reduced_shape(), n_req=3),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("top_k,sink,local", [(8, 1, 2), (1, 0, 1), (20, 2, 4)])
def test_sparse_steps(name, top_k, sink, local):
    case = CASES[name]()
    n = len(case.lens)
    pred = make_predictor(case, max_seq_len=int(case.lens.max()) + 40, keep=True)
    pred.sparse_steps(top_k, sink, local)
    pred.prefill(list(range(n)), case.lens, *device_states(case))
    check_block_keys(read(pred, case))
    slots = list(range(n))
    for t in range(1, 20):
        if t == 12:
            slots = [2, 0]
        S = [x[slots].contiguous() for x in device_states(case, step_inputs(case, t))]
        z, _ = pred.step(slots, *S)
        assert z.isfinite().all()
        if t in (1, 4, 5, 12, 16, 17, 19):
            check_step(pred, case, slots, top_k, sink, local)
    say(f"  {name}: {n} requests, top_k {top_k}")
    pred.close()


def test_short_caches_and_off_keep_their_bits():
    """No request above top_k pages, then some above, then turned off: against
    a context without sparse steps."""
    case = make_case(1, lens=[100, 60, 127, 5], shape=reduced_shape(), n_req=4)
    a, b = (make_predictor(case, max_seq_len=400) for _ in range(2))
    a.sparse_steps(8, 1, 2)
    H = device_states(case)
    assert torch.equal(a.prefill(range(4), case.lens, *H)[0], b.prefill(range(4), case.lens, *H)[0])
    for t in range(1, 6):
        S = device_states(case, step_inputs(case, t))
        (za, ha), (zb, hb) = (p.step(range(4), *S, want_hdraft=True) for p in (a, b))
        # the third request (127 tokens) takes its ninth page with the second step
        same = torch.equal(ha, hb) and torch.equal(za, zb)
        if t == 1:
            assert same
            with pytest.raises(B.OutletsError):
                a.buffer("SELECTED", torch.int32)
        elif t == 2:
            # a request with at most top_k pages reads all of its tokens: the
            # same sums in another order and split
            assert not same
            for i in (0, 1, 3):
                d = (ha[i].float() - hb[i].float()).norm() / hb[i].float().norm()
                assert d <= 2e-2
            break
    a.sparse_steps(0)
    a.release(range(4)), b.release(range(4))
    a.prefill(range(4), case.lens, *H), b.prefill(range(4), case.lens, *H)
    for t in range(1, 5):
        S = device_states(case, step_inputs(case, t))
        (za, ha), (zb, hb) = (p.step(range(4), *S, want_hdraft=True) for p in (a, b))
        assert torch.equal(za, zb) and torch.equal(ha, hb)
    with pytest.raises(B.OutletsError):
        a.buffer("BLOCK_KEYS", torch.bfloat16)
    a.close(), b.close()


def test_noalloc_and_reused_pages():
    """The no-allocation step takes the same selection and bits; pages that
    return through release get new block keys."""
    case = make_case(1, lens=[600, 40, 900], shape=reduced_shape(), n_req=3, attn_gate=True)
    a, b = (make_predictor(case, max_seq_len=1000) for _ in range(2))
    for p in (a, b):
        p.sparse_steps(10, 1, 3)
        p.sparse_steps(6, 1, 2)                      # again: the new sizes hold
    H = device_states(case)
    for turn in range(2):
        for p in (a, b):
            p.prefill([0, 1, 2] if turn == 0 else [2, 0, 1], case.lens, *H)
        for t in range(1, 4):
            S = device_states(case, step_inputs(case, t))
            za, ha = a.step([0, 2], *[x[:2] for x in S], want_hdraft=True)
            zb, hb = b.step([0, 2], *[x[:2] for x in S], want_hdraft=True, noalloc=True)
            assert torch.equal(za, zb) and torch.equal(ha, hb)
        r = read(a, case)
        check_block_keys(r)
        sel = a.buffer("SELECTED", torch.int32).view(2, 2, 6)
        # each request's newest page is the last of its list
        assert sel.amax(dim=2).tolist() == [[(r["len"][s] - 1) // PAGE] * 2 for s in (0, 2)]
        for p in (a, b):
            p.release([0, 1, 2])
    a.close(), b.close()


def test_refusals():
    case = make_case(0)
    pred = make_predictor(case)
    for args in ((4, -1, 1), (4, 1, 0), (4, 3, 2), (-1, 0, 1), (2**31 - 1, 2**31 - 1, 2**31 - 1)):
        with pytest.raises(B.OutletsError) as e:
            pred.sparse_steps(*args)
        assert e.value.rc == B.OUTLETS_ERR_INVALID_ARG
    pred.prefill(range(len(case.lens)), case.lens, *device_states(case))
    with pytest.raises(B.OutletsError) as e:
        pred.sparse_steps(4, 1, 1)
    assert e.value.rc == B.OUTLETS_ERR_SLOT_BUSY
    pred.sparse_steps(0)
    pred.release(range(len(case.lens)))
    pred.sparse_steps(4, 1, 1)
    pred.close()
