"""Attention over the 4-bit K/V cache where the numbers span wide ranges: value
scales, scores, windows and queries at the ends of what the formats hold, in
the kernel for few query rows and in the one for many.  Tolerances as in
test_gpu_kv4, except where a test derives its own."""
import numpy as np
import pytest

from oracle import q4
from test_gpu_kv4 import PAGE, check_attention, dev, i32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


def v_params(data, D):
    """The params of the values: a view [..][D / 64][64] of the blocks' ends."""
    at = PAGE * D + (D // 64) * PAGE * 2
    return data[..., at:].view(np.uint16).reshape(data.shape[:-1] + (D // 64, PAGE))


def scale_bits(exponent):
    return int(np.float16(2.0 ** exponent).view(np.uint16))


def attend(tq, c, q, slots, n, layer=0, **kw):
    import torch
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    tq.tq_kv4_attention(q, c, layer, i32(slots), i32(np.concatenate([[0], np.cumsum(n)])), out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    c.check()
    return out, lse


def queries(rng, T, Hq, D, dtype, positive=False):
    import torch
    q = rng.standard_normal((T, Hq, D)).astype(np.float32)
    return dev(np.abs(q) if positive else q).to({"fp16": torch.float16, "bf16": torch.bfloat16}[dtype])


# ------------------------------------------------------------- value scales
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("large,small", [(0, 1), (1, 0)])
@pytest.mark.parametrize("lengths,n,heads,group", [([500, 70], [1, 1], 2, 4), ([500, 70], [5, 3], 2, 4), ([9000], [2], 1, 3),
                                                   ([330, 260], [170, 60], 4, 8)])
def test_a_group_of_small_values_beside_large_ones(tq, dtype, large, small, lengths, n, heads, group):
    """One group of a head's dimensions at 2^12, the other at 2^-16."""
    D = 128
    c, data, table, length, _ = make(tq, lengths, heads, D, seed=51, poison=False)
    p = v_params(data, D)
    for gr, e in ((large, 12), (small, -16)):
        p[..., gr, :] = p[..., gr, :] & 15 | scale_bits(e)
    c.data.copy_(dev(data))
    q = queries(np.random.default_rng(52), sum(n), heads * group, D, dtype)
    out, lse = attend(tq, c, q, range(len(n)), n)
    check_attention(c, data, table, length, range(len(n)), n, heads, group, D, 0, q, out, lse, True, 0, D ** -0.5, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("far", [2.3, 4.6, 0.0])
@pytest.mark.parametrize("at", [0, 130, 298])
def test_a_token_of_large_values_that_counts_little(tq, D, dtype, far, at):
    """Values of 2^12 at one token whose probability is about 2^-30 or 2^-60 of the
    others' (far > 0) or ordinary, everything else at 2^-16; with at = 298 two of the
    three queries do not see it."""
    heads, group = 2, 4
    c, data, table, length, _ = make(tq, [300], heads, D, seed=53, poison=False)
    p = v_params(data, D)
    p[...] = p & 15 | scale_bits(-16)
    rng = np.random.default_rng(54)
    for h in range(heads):
        q4.store(data[0, table[0, at // PAGE], h], D, at % PAGE, np.full(D, -far * (128 / D) ** 0.5, np.float32),
                 (rng.standard_normal(D) * 10000).astype(np.float32))
    c.data.copy_(dev(data))
    for n in (1, 3):
        q = queries(rng, n, heads * group, D, dtype, positive=True)
        out, lse = attend(tq, c, q, [0], [n])
        check_attention(c, data, table, length, [0], [n], heads, group, D, 0, q, out, lse, True, 0, D ** -0.5, dtype)


def test_zero_scales_and_growing_scores(tq):
    """Groups whose values are all zero keep nothing of a row's references; scores
    that grow along the sequence move them many times."""
    D, heads, group = 128, 2, 4
    rng = np.random.default_rng(55)
    c, data, table, length, _ = make(tq, [700], heads, D, seed=56, poison=False)
    ramp = np.linspace(0, 40, 700)
    for h in range(heads):
        for t in range(700):
            v = rng.standard_normal(D).astype(np.float32) * 2.0 ** rng.integers(-14, 10)
            v[:64] *= t % 3 > 0
            v[64:] *= t > 350
            q4.store(data[0, table[0, t // PAGE], h], D, t % PAGE,
                     (rng.standard_normal(D) + ramp[t] / 10).astype(np.float32), v)
    c.data.copy_(dev(data))
    for n in (1, 4):
        q = queries(rng, n, heads * group, D, "fp16", positive=True)
        for kw in ({}, {"scale": -0.05}):
            out, lse = attend(tq, c, q, [0], [n], **kw)
            check_attention(c, data, table, length, [0], [n], heads, group, D, 0, q, out, lse, True, 0,
                            kw.get("scale", D ** -0.5), "fp16")


# ------------------------------------------------------------------- scores
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,n,heads,group", [(400, 1, 2, 4), (400, 5, 2, 4), (30000, 1, 1, 4), (400, 210, 4, 8)])
def test_scores_of_ten_digits(tq, dtype, D, L, n, heads, group):
    """Scores up to 2^34, exact in float32 and at least 2^24 apart or equal: a row's
    output is the mean of the values of its best keys, which repeat.  The
    probabilities are 0 and 1, so of test_gpu_kv4's tolerance what remains is the
    output's rounding, P's (2^-11 a) and the sums' (2^-17 a)."""
    import torch
    rng = np.random.default_rng(57)
    c, data, table, length, _ = make(tq, [L], heads, D, seed=58, poison=False)
    kp = data[..., PAGE * D:PAGE * D + (D // 64) * PAGE * 2].view(np.uint16)
    kp[...] = scale_bits(10) | 8
    few = rng.integers(0, 256, (6, heads, D // 2)).astype(np.uint8)  # six different keys
    for t in range(L):
        for h in range(heads):
            data[:, table[0, t // PAGE], h, t % PAGE * (D // 2):(t % PAGE + 1) * (D // 2)] = few[t * 7 % 6 if t % 5 else 0, h]
    c.data.copy_(dev(data))
    q = rng.choice([-16384.0, 0.0, 16384.0], (n, heads * group, D)).astype(np.float32)
    q = dev(q).to({"fp16": torch.float16, "bf16": torch.bfloat16}[dtype])
    out, lse = attend(tq, c, q, [0], [n], scale=1.0)
    got, gl, qf = out.float().cpu().numpy(), lse.cpu().numpy(), q.float().cpu().numpy().astype(np.float64)
    for h in range(heads):
        K, V = q4.sequence(data, table, length, 0, 0, h, D)
        for hq in range(h * group, (h + 1) * group):
            s = qf[:, hq] @ K.T
            for i in range(n):
                end = L - n + i + 1
                best = np.flatnonzero(s[i, :end] == s[i, :end].max())
                o, a = V[best].mean(0), np.abs(V[best]).mean(0)
                tol = np.abs(o) * 2.0 ** (-11 if dtype == "fp16" else -8) + (2.0 ** -11 + 2.0 ** -17) * a + 2.0 ** -24
                assert np.all(np.abs(got[i, hq] - o) <= tol), (h, hq, i, got[i, hq][:4], o[:4])
                m = s[i, :end].max()
                assert abs(gl[i, hq] - (m + np.log(len(best)))) <= 2.0 ** -21 * abs(m) + 2.0 ** -17


# ------------------------------------------------------------------ windows
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30, 2 ** 31 - 64])
@pytest.mark.parametrize("lengths,n,heads,group", [([2, 0, 100, 1], [9, 3, 4, 70], 2, 4), ([2, 0, 100, 1], [210, 70, 4, 99], 4, 8)])
def test_windows_wider_than_any_sequence(tq, window, lengths, n, heads, group):
    """More queries than tokens below the widest windows there are."""
    D = 128
    c, data, table, length, _ = make(tq, lengths, heads, D, seed=59)
    q = queries(np.random.default_rng(60), sum(n), heads * group, D, "fp16")
    out, lse = attend(tq, c, q, range(4), n, window=window)
    check_attention(c, data, table, length, range(4), n, heads, group, D, 0, q, out, lse, True, window, D ** -0.5, "fp16")


# ------------------------------------------------------------------ queries
@pytest.mark.parametrize("e", [-126, -110, 75, 90, 124])
@pytest.mark.parametrize("L,n,heads,group", [(300, 2, 2, 4), (300, 200, 4, 8)])
def test_bf16_queries_of_every_size(tq, e, L, n, heads, group):
    """Queries around 2^e with a scale that brings the scores back to ordinary ones."""
    import torch
    D = 128
    c, data, table, length, _ = make(tq, [L], heads, D, seed=61)
    q = np.clip(np.random.default_rng(62).standard_normal((n, heads * group, D)), -7, 7) * 2.0 ** e
    q = dev(q.astype(np.float32)).to(torch.bfloat16)
    scale = float(np.float32(2.0 ** max(-e, -126) * D ** -0.5))
    out, lse = attend(tq, c, q, [0], [n], scale=scale)
    check_attention(c, data, table, length, [0], [n], heads, group, D, 0, q, out, lse, True, 0, scale, "bf16")


# --------------------------------------------------------------------- joins
@pytest.mark.parametrize("lengths,n", [([300], [1]), ([5000, 1, 0], [1, 1, 1]), ([20000], [2]), ([64] * 40, [1] * 40)])
def test_every_worker_says_what_there_is_to_join(tq, lengths, n):
    """The kernel that joins parts reads an entry of every worker: after a call on
    scratch memory full of ones each names workers that exist, or none."""
    import ctypes
    import torch
    D, heads, group = 128, 2, 4
    c, *_ = make(tq, lengths, heads, D, seed=63)
    T, L = sum(n), tq.lib()
    q = torch.randn((T, heads * group, D), device="cuda").half()
    out, slots, indptr = torch.empty_like(q), i32(range(len(n))), i32(np.concatenate([[0], np.cumsum(n)]))
    nbytes = L.tq_kv4_attention_workspace_bytes(c._ref, len(n), T, max(n), heads * group)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    assert L.tq_kv4_attention(c._ref, 0, len(n), p(slots), p(indptr), T, max(n), heads * group, 0, p(q), heads * group * D,
                              D ** -0.5, 1, 0, p(out), heads * group * D, None, p(ws), nbytes, p(c.status), None) == 0
    torch.cuda.synchronize()
    c.check()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    workers = sms * 12 if max(n) * group <= 8 else sms * 8  # warps of the chip; an entry is 48 bytes, its second word the last worker
    entries = ws[:workers * 48].view(torch.int32).view(workers, 12).cpu().numpy()
    some = entries[:, 1] >= 0
    assert np.all(entries[:, 1] >= -1) and np.all(entries[:, 1] < workers)
    assert np.all(entries[some, 0] >= 0) and np.all(entries[some, 0] < entries[some, 1])
    assert np.all(entries[some, 7] < T) and np.all(entries[some, 8] < heads)
