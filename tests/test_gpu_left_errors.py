"""A HIP error that an earlier call of the thread left (a failed allocation) is
not reported by calls whose own work is queued."""
import ctypes as C

import pytest
import torch

from gpu_common import device_states, make_case, make_predictor, reduced_shape, require_gpu, step_inputs
from paper_2609_01068_amd import binding as B
from test_gpu_paged import Serving, i32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def leave_error():
    """An allocation that no device has room for, its error unread."""
    p = C.c_void_p()
    assert B.lib().hipMalloc(C.byref(p), C.c_size_t(1 << 50)) != 0 and not p.value


def test_paged_cache_calls_after_an_error():
    s = Serving()
    n_kv, G, hd = s.shape
    leave_error()
    s.pt.reset()
    for i in range(2):
        qkv = randn((40, (G + 2) * n_kv * hd), "bf16", i)
        slots, new = i32([0, 2]), i32([30 - 20 * i, 9])
        q, k, v = (t.view(40, -1, hd) for t in qkv.split([n_kv * G * hd, n_kv * hd, n_kv * hd], dim=1))
        leave_error()
        rows = s.pt.append(slots, new, 40)
        assert rows.status[0].item() == 0
        leave_error()
        s.kv.write(rows.slot_map, k, v)
        leave_error()
        sel = s.kv.select(q, rows.row_slot, rows.positions, s.top_k, 1, 2)
        leave_error()
        out = s.kv.attend(q, rows.row_slot, rows.positions, sel)
        s.check(rows, sel, out, qkv)
    leave_error()
    assert s.pt.release(i32([0])).item() == 0
    assert s.pt.seq_len.tolist() == [0, 0, 18, 0, 0, 0]


def test_predict_calls_after_a_failed_allocation():
    """Sparse steps whose selection no device can hold are refused, and off: the
    context then answers as one that never asked for them."""
    case = make_case(1, lens=[100, 60, 127], shape=reduced_shape(), n_req=3)
    a, b = (make_predictor(case, max_seq_len=400, max_batch_requests=4096, max_slots=4096, num_pages=4096)
            for _ in range(2))
    # 4 bytes, 4,096 requests, 2 KV heads and 2^31 - 1 pages: 64 TiB
    with pytest.raises(B.OutletsError) as e:
        a.sparse_steps(2**31 - 1, 1, 4)
    assert e.value.rc == B.OUTLETS_ERR_NOMEM
    H = device_states(case)
    assert torch.equal(a.prefill(range(3), case.lens, *H)[0], b.prefill(range(3), case.lens, *H)[0])
    for t in range(1, 4):
        S = device_states(case, step_inputs(case, t))
        leave_error()
        za, ha = a.step(range(3), *S, want_hdraft=True, noalloc=t == 2)
        zb, hb = b.step(range(3), *S, want_hdraft=True)
        assert torch.equal(za, zb) and torch.equal(ha, hb)
    assert a.meta(B.OUTLETS_META_SEQ_LEN)[:3].tolist() == [103, 63, 130]
    a.release(range(3))
    a.sparse_steps(4, 1, 1)                          # and a size that fits is taken
    a.prefill(range(3), case.lens, *H)
    a.step(range(3), *device_states(case, step_inputs(case, 1)))
    assert a.buffer("SELECTED", torch.int32).numel() == 3 * 2 * 4
    a.close(), b.close()


def test_a_refused_size_holds_no_memory():
    """What was allocated before the allocation that failed is freed."""
    case = make_case(1, lens=[100, 60, 127], shape=reduced_shape(), n_req=3)
    pred = make_predictor(case, max_seq_len=400, max_batch_requests=4096, max_slots=4096, num_pages=200000)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    with pytest.raises(B.OutletsError):
        pred.sparse_steps(2**31 - 1, 1, 4)           # its block keys alone take 102 MB
    assert torch.cuda.mem_get_info()[0] == free
    pred.close()
