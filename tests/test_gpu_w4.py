"""4-bit weights on the GPU against their definition in numpy.

y's tolerance: with T = sum |x| (|scale| c + |minimum|), every fp32 addition
costs at most 2^-23 of what is added up (tensor-core sums truncate); a row's sum
takes 8 per group in the tensor cores, one per group and a few to join the
parts: 2^-23 (16 + K / 128 + 32) T, and 2^-11 |y| for fp16 results (2^-25 below
its normal range)."""
import numpy as np
import pytest

from oracle import q4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def weights(N, K, seed):
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    s = np.exp(rng.normal(-4, 1, (N, K // 128))).astype(np.float16)
    m = (s.astype(np.float32) * rng.normal(-7.5, 2, s.shape)).astype(np.float16)
    return codes, s, m


def check(tq, M, N, K, seed=0, f32=False, xs=1.0, edit=None):
    import torch
    codes, s, m = weights(N, K, seed)
    if edit:
        edit(codes, s, m)
    x = (np.random.default_rng(seed + 1).standard_normal((M, K)) * xs).astype(np.float16)
    w = tq.pack_w4(dev(codes), dev(s), dev(m))
    y = tq.tq_w4_linear(dev(x), w, f32=f32)
    torch.cuda.synchronize()
    W = q4.w4_values(codes, s, m)
    xf = x.astype(np.float64)
    ref = xf @ W.T
    T = np.abs(xf) @ (np.repeat(np.abs(s.astype(np.float64)), 128, 1) * codes +
                      np.repeat(np.abs(m.astype(np.float64)), 128, 1)).T
    tol = 2.0 ** -23 * (16 + K // 128 + 32) * T + (0 if f32 else 2.0 ** -11 * np.abs(ref) + 2.0 ** -25)
    err = np.abs(y.float().cpu().numpy() - ref)
    assert y.dtype == (torch.float32 if f32 else torch.float16)
    assert np.all(err <= tol), (float((err / tol).max()), np.argwhere(~(err <= tol))[:4])
    return w, codes, s, m


@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 17, 31, 40, 65, 130])
@pytest.mark.parametrize("N,K", [(1, 128), (15, 256), (33, 640), (200, 1408)])
def test_shapes(tq, M, N, K):
    check(tq, M, N, K, seed=M + N, f32=bool(M & 1))


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (1, 40007, 1024), (5, 1000, 12288), (16, 9725, 2560), (40, 3000, 4096),
                                   (2, 64, 65536)])
def test_larger(tq, M, N, K):
    check(tq, M, N, K, f32=M == 1)


def test_activations_of_every_size(tq):
    for xs in (1e-6, 1e-3, 300.0, 4000.0):
        check(tq, 3, 100, 512, seed=5, f32=True, xs=xs)


def test_scales_at_the_ends(tq):
    def edit(codes, s, m):
        s[0], m[0] = 0.0, 1.5             # a constant group
        s[1], m[1] = 2.0 ** -24, 0.0      # fp16's smallest
        s[2], m[2] = -0.25, 3.0           # falling codes
        s[3], m[3] = 1000.0, -7500.0
    check(tq, 4, 20, 384, f32=True, edit=edit)


def test_not_a_number_stays_in_its_row_and_token(tq):
    import torch
    codes, s, m = weights(50, 512, 3)
    s[7, 2] = np.inf
    m[9, 0] = np.nan
    x = np.random.default_rng(4).standard_normal((5, 512)).astype(np.float16)
    x[2, 100], x[3, 5] = np.inf, np.nan
    w = tq.pack_w4(dev(codes), dev(s), dev(m))
    y = tq.tq_w4_linear(dev(x), w).float().cpu().numpy()
    good = np.ones((5, 50), bool)
    good[:, [7, 9]] = False
    good[[2, 3]] = False
    assert np.isfinite(y[good]).all()
    assert np.isnan(y[:, 9]).all() and np.isnan(y[3]).all() and not np.isfinite(y[:, 7]).any()
    assert not np.isfinite(y[2]).any()


def test_quantize_is_round_to_nearest(tq):
    import torch
    rng = np.random.default_rng(8)
    W = (rng.standard_normal((70, 640)) * np.exp(rng.normal(-4, 1, (70, 1)))).astype(np.float16)
    W[3, :128] = 0.5
    W[4, 128:256] = 0
    codes, s, m = q4.w4_quantize(W)
    a, b = tq.quantize_w4(dev(W)), tq.pack_w4(dev(codes), dev(s), dev(m))
    assert torch.equal(a.tiles, b.tiles)
    D = tq.tq_w4_dequantize(a)
    assert np.array_equal(D.cpu().numpy(), q4.w4_values(codes, s, m).astype(np.float32).astype(np.float16))
    W[5, 7] = np.nan
    with pytest.raises(tq.TQError):
        tq.quantize_w4(dev(W))
    w = tq.quantize_w4(dev(W), check=False)
    D = tq.tq_w4_dequantize(w).cpu().numpy()
    assert np.isnan(D[5, :128]).all() and np.isfinite(D[5, 128:]).all()


def test_pack_reports_codes(tq):
    codes, s, m = weights(10, 128, 1)
    codes[3, 5] = 16
    with pytest.raises(tq.TQError):
        tq.pack_w4(dev(codes), dev(s), dev(m))


def test_refusals(tq):
    import torch
    codes, s, m = weights(10, 256, 1)
    w = tq.pack_w4(dev(codes), dev(s), dev(m))
    x = torch.zeros((2, 256), device="cuda").half()
    for f in (lambda: tq.tq_w4_linear(x.float(), w), lambda: tq.tq_w4_linear(x[:, :128], w),
              lambda: tq.tq_w4_linear(x, w, y=torch.zeros((2, 10), device="cuda")),
              lambda: tq.tq_w4_linear(x, w, y=torch.zeros((1, 10), device="cuda").half()),
              lambda: tq.tq_w4_linear(x.t().contiguous().t(), w),
              lambda: tq.pack_w4(dev(codes), dev(s[:, :1]), dev(m)), lambda: tq.pack_w4(dev(codes).int(), dev(s), dev(m))):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(tq.TQError):
        tq.tq_w4_linear(x, w, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(tq.TQError):
        tq.quantize_w4(torch.zeros((4, 100), device="cuda").half())


def test_same_bits_again_on_streams_and_in_a_graph(tq):
    import torch
    codes, s, m = weights(3000, 2048, 1)
    w = tq.pack_w4(dev(codes), dev(s), dev(m))
    x = torch.randn((3, 2048), device="cuda").half()
    ref = tq.tq_w4_linear(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(ref) for _ in range(6)]
    ws = [tq.workspace(int(tq.lib().tq_w4_workspace_bytes(3, 3000, 2048)), "cuda") for _ in outs]
    for i, (o, b) in enumerate(zip(outs, ws)):
        tq.tq_w4_linear(x, w, y=o, ws=b, stream=side if i % 2 else None)
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_w4_linear(x, w, y=outs[0], ws=ws[0])
    x.mul_(0.5)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], tq.tq_w4_linear(x, w))
