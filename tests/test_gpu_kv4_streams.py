"""The 4-bit K/V cache's and the 4-bit weights' calls in graphs and on streams
other than the current one: whose memory they use, and in what order."""
import numpy as np
import pytest

from test_gpu_kv4 import dev, i32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


# ------------------------------------------------------------------- graphs
def attention_step(tq, lengths, n, heads, group, D, seed):
    """(call, output) of an attention call with buffers of its own."""
    import torch
    c, *_ = make(tq, lengths, heads, D, seed=seed)
    q = torch.randn((sum(n), heads * group, D), device="cuda").half()
    out = torch.empty_like(q)
    slots, indptr = i32(range(len(n))), i32(np.concatenate([[0], np.cumsum(n)]))
    return c, lambda **kw: tq.tq_kv4_attention(q, c, 0, slots, indptr, max_q=max(n), out=out, **kw), out


def test_graphs_do_not_share_scratch_memory(tq, monkeypatch):
    """Two graphs of one cache (different shapes, as a server captures them for its
    batch sizes) and an eager call have scratch memory of their own; replayed side
    by side on two streams they give the eager results."""
    import torch
    c, *_ = make(tq, [9000, 700, 3000], 2, 128, seed=1)
    used = []
    scratch = tq.Kv4Cache._scratch

    def spy(self, *args):
        ws = scratch(self, *args)
        used.append((ws.data_ptr(), ws.numel()))
        return ws
    monkeypatch.setattr(tq.Kv4Cache, "_scratch", spy)
    calls = []
    for slots in ([0, 1, 2], [2, 0]):
        q = torch.randn((len(slots), 8, 128), device="cuda").half()
        out = torch.empty_like(q)
        s, ip = i32(slots), i32(range(len(slots) + 1))
        calls.append((lambda q=q, out=out, s=s, ip=ip: tq.tq_kv4_attention(q, c, 0, s, ip, max_q=1, out=out), out))
    refs = []
    for call, out in calls:
        call()
        refs.append(out.clone())
    eager = set(used)
    used.clear()
    graphs = []
    for call, out in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    blocks = sorted(eager | set(used))
    assert len(blocks) >= 3 and len(set(used)) == 2
    for (a, n), (b, _) in zip(blocks, blocks[1:]):
        assert a + n <= b, "scratch memory of two graphs, or of a graph and an eager call, overlaps"
    for _, out in calls:
        out.zero_()
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(50):
        for g, s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    c.check()
    for (_, out), ref in zip(calls, refs):
        assert torch.equal(out, ref)


def test_callers_workspace(tq):
    import torch
    c, call, out = attention_step(tq, [500, 90], [1, 1], 2, 4, 128, seed=2)
    call()
    ref = out.clone()
    L = tq.lib()
    n = L.tq_kv4_attention_workspace_bytes(c._ref, 2, 2, 1, 8)
    ws = tq.workspace(n, "cuda")
    out.zero_()
    call(ws=ws)
    assert torch.equal(out, ref)
    for bad in (ws[:n - 256], ws[16:]):
        with pytest.raises(tq.TQError):
            call(ws=bad)
    with pytest.raises(ValueError):
        call(ws=ws.view(torch.int32))
    e = tq.workspace(L.tq_kv4_extend_workspace_bytes(c._ref, 1, 3), "cuda")
    indptr, where = tq.tq_kv4_extend(c, i32([1]), i32([3]), 3, ws=e)
    assert indptr.tolist() == [0, 3] and int(where.min()) >= 0
    with pytest.raises(tq.TQError):
        tq.tq_kv4_extend(c, i32([1]), i32([3]), 3, ws=e[:e.numel() - 1])
    m = tq.workspace(L.tq_kv4_compact_workspace_bytes(c._ref), "cuda")
    remap, live = tq.tq_kv4_compact(c, ws=m)
    assert int(live) == 8 + 2
    with pytest.raises(tq.TQError):
        tq.tq_kv4_compact(c, ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    c.check()
