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


# ------------------------------------------------------------------ streams
def stream_of(t):
    """The stream whose memory a tensor lives in."""
    import torch
    p = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= p < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's memory")


def test_memory_comes_from_the_stream_that_uses_it(tq):
    """Memory freed on the current stream may still be in use there: what a call on
    another stream allocates has to be that stream's."""
    import torch
    c, *_ = make(tq, [300, 70], 2, 128, seed=3)
    q = torch.randn((2, 8, 128), device="cuda").half()
    W, x = torch.randn((64, 256), device="cuda").half(), torch.randn((2, 256), device="cuda").half()
    codes, s, m = torch.ones((64, 256), dtype=torch.uint8, device="cuda"), W[:, :2].contiguous(), W[:, 2:4].contiguous()
    slots, ip, one = i32([0, 1]), i32([0, 1, 2]), i32([1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = tq.tq_kv4_attention(q, c, 0, slots, ip, max_q=1, stream=side)
    indptr, where = tq.tq_kv4_extend(c, slots, one, 2, stream=side)
    k, v = tq.tq_kv4_read(c, 0, where, stream=side)
    remap, live = tq.tq_kv4_compact(c, stream=side)
    a, b = tq.quantize_w4(W, stream=side), tq.pack_w4(codes, s, m, stream=side)
    y, D = tq.tq_w4_linear(x, a, stream=side), tq.tq_w4_dequantize(a, stream=side)
    torch.cuda.synchronize()
    c.check()
    for t in (out, indptr, where, k, v, remap, live, a.tiles, b.tiles, y, D, *c._ws.values()):
        assert stream_of(t) == side.cuda_stream
    assert stream_of(q) == torch.cuda.current_stream().cuda_stream


def test_errors_reported_on_another_stream_are_seen(tq):
    """The reports of work that is still under way on another stream."""
    import torch
    c, *_ = make(tq, [100], 2, 128, seed=4)
    k = torch.ones((1, 2, 128), device="cuda").half()
    W = torch.full((16, 128), float("nan"), device="cuda").half()
    codes, s = torch.full((16, 128), 16, dtype=torch.uint8, device="cuda"), torch.ones((16, 1), device="cuda").half()
    beyond = i32([c.pages * 64])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for call in (lambda: tq.quantize_w4(W, stream=side), lambda: tq.pack_w4(codes, s, s, stream=side)):
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)  # about 50 ms
        with pytest.raises(tq.TQError):
            call()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    tq.tq_kv4_append(k, k, c, 0, beyond, stream=side)
    with pytest.raises(tq.TQError):
        c.check()
    c.check()
