"""Empty batches of the 4-bit K/V cache's calls: nothing to do, and no error."""
import pytest

from test_gpu_kv4 import i32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


@pytest.mark.parametrize("D", [64, 128])
def test_empty_lists(tq, D):
    import torch
    c, *_ = make(tq, [100, 0, 70], 2, D, seed=1)
    before = [x.clone() for x in (c.data, c.table, c.length, c.refs)]
    none = i32([])
    indptr, where = tq.tq_kv4_extend(c, none, none, 0)
    assert indptr.tolist() == [0] and where.shape == (0,)
    for T in (0, 3):  # tokens that belong to no sequence are not written
        q = torch.ones((T, 8, D), device="cuda").half()
        out = torch.full_like(q, 7.0)
        tq.tq_kv4_attention(q, c, 0, none, indptr, out=out)
        assert bool((out == 7.0).all())
    tq.tq_kv4_fork(c, none, none)
    tq.tq_kv4_free(c, none)
    tq.tq_kv4_free(c, none, none)
    tq.tq_kv4_copy_pages(c, c, none, none)
    k = torch.ones((0, 2, D), device="cuda").half()
    tq.tq_kv4_append(k, k, c, 0, none)
    K, V = tq.tq_kv4_read(c, 0, none)
    assert K.shape == V.shape == (0, 2, D)
    c.check()
    assert all(torch.equal(a, b) for a, b in zip(before, (c.data, c.table, c.length, c.refs)))
    # no sequence can have the tokens that the call says there are
    indptr, where = tq.tq_kv4_extend(c, none, none, 5)
    assert indptr.tolist() == [0] and where.tolist() == [-1] * 5 and int(c.status.item()) == 128
    c.status.zero_()


def test_a_captured_step_without_sequences(tq):
    import torch
    c, *_ = make(tq, [100], 2, 128, seed=2)
    none, q = i32([]), torch.zeros((0, 8, 128), device="cuda").half()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        indptr, where = tq.tq_kv4_extend(c, none, none, 0)
        tq.tq_kv4_attention(q, c, 0, none, indptr)
    g.replay()
    torch.cuda.synchronize()
    c.check()
    assert indptr.tolist() == [0]


def test_negative_counts_are_refused(tq):
    import ctypes
    c, *_ = make(tq, [100], 2, 128, seed=3)
    L, p = tq.lib(), ctypes.c_void_p(c.status.data_ptr())
    assert L.tq_kv4_fork(c._ref, -1, None, None, p, None) == -2
    assert L.tq_kv4_free(c._ref, -1, None, None, p, None) == -2
    assert L.tq_kv4_fork(c._ref, 1, None, None, p, None) == -1
    assert L.tq_kv4_extend_workspace_bytes(c._ref, -1, 0) == 0 < L.tq_kv4_extend_workspace_bytes(c._ref, 0, 0)
