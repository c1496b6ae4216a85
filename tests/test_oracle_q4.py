"""The 4-bit definitions on the CPU: what a code stands for, and the host
checks of the entry points that take them (no GPU)."""
import ctypes

import numpy as np
import pytest

from oracle import q4


def groups():
    rng = np.random.default_rng(3)
    yield rng.standard_normal(64)
    yield rng.standard_normal(64) * 1e-3 + 4.0       # far from zero: zero stays on the grid
    yield -np.abs(rng.standard_normal(64)) - 2.0
    yield np.zeros(64)
    yield np.full(64, 3.5)
    yield rng.standard_normal(64) * 6e-7             # subnormal fp16
    yield rng.standard_normal(64) * 6000.0
    x = np.zeros(64)
    x[17] = 1.0
    yield x


@pytest.mark.parametrize("i", range(8))
def test_values_are_fp16_numbers_within_half_a_step(i):
    x = np.asarray(list(groups())[i], np.float16)
    codes, param = q4.encode(x.astype(np.float32))
    v = q4.decode(codes, param)
    assert np.array_equal(v.astype(np.float16).astype(np.float64), v)  # exact in fp16
    s = float(np.uint16(param & 0xFFF0).view(np.float16))
    # the step is at most 2^-6 wider than the range asks for (seven bits, rounded up)
    # plus one unit where it is subnormal; the zero's own rounding shifts the ends by half a step
    span = max(0.0, float(x.max())) - min(0.0, float(x.min()))
    assert s <= span / 15 * (1 + 2 ** -6 + 2 ** -10) + 16 * 2.0 ** -24
    assert np.all(np.abs(v - x.astype(np.float64)) <= s * (1 + 2 ** -9))
    inner = (codes > 0) & (codes < 15)
    assert np.all(np.abs(v - x.astype(np.float64))[inner] <= s * (0.5 + 2 ** -9))
    assert q4.encode(np.zeros(64, np.float32))[1] == 0


def test_groups_that_cannot_be_held_are_nan():
    for bad in (np.inf, -np.inf, np.nan, 65504.0):
        x = np.ones(64, np.float32)
        x[5], x[6] = bad, -60000.0
        codes, param = q4.encode(x)
        assert np.all(np.isnan(q4.decode(codes, param)))
    codes, param = q4.encode(np.full(64, 50000.0, np.float32))
    assert np.all(np.isfinite(q4.decode(codes, param)))


def test_store_and_block_values_agree():
    rng = np.random.default_rng(5)
    for D in (64, 128):
        block = rng.integers(0, 256, q4.block_bytes(D)).astype(np.uint8)
        k, v = (rng.standard_normal(D).astype(np.float16).astype(np.float32) for _ in "kv")
        q4.store(block, D, 37, k, v)
        K, V = q4.block_values(block, D)
        for x, got in ((k, K[37]), (v, V[37])):
            want = np.concatenate([q4.decode(*q4.encode(x[g:g + 64])) for g in range(0, D, 64)])
            assert np.array_equal(got, want)


def cache(tq, **kw):
    c = tq.tq_kv4_cache(2, 10, 2, 128, 4, 8, 0x1000, 0x1000, 0x1000, 0x1000)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def test_cache_argument_errors_without_gpu():
    from paper_2609_09240_gb300 import tq
    L = tq.lib()
    assert L.tq_kv4_block_bytes(128) == 8704 and L.tq_kv4_block_bytes(64) == 4352 and L.tq_kv4_block_bytes(96) == 0
    P = 0x1000
    att = lambda c, layer=0, count=1, tokens=1, max_q=1, heads=4, dt=0, q=P, qs=512, sc=1.0, causal=1, window=0, out=P, \
        os_=512, ws=P, nws=1 << 30: L.tq_kv4_attention(c, layer, count, P, P, tokens, max_q, heads, dt, q, qs, sc, causal,
                                                      window, out, os_, None, ws, nws, P, None)
    assert att(None) == -1
    for kw in (dict(layers=0), dict(pages=0), dict(pages=(1 << 24) + 1), dict(heads=0), dict(dim=96), dict(slots=0),
               dict(max_pages=0)):
        assert att(cache(tq, **kw)) == -2, kw
    for name in ("data", "table", "length", "refs"):
        assert att(cache(tq, **{name: None})) == -1
    assert att(cache(tq, data=0x1008)) == -3 and att(cache(tq, table=0x1002)) == -3
    ok = cache(tq)
    for kw in (dict(layer=2), dict(layer=-1), dict(count=0), dict(tokens=-1), dict(max_q=2), dict(heads=3), dict(heads=0),
               dict(dt=2), dict(qs=511), dict(qs=516), dict(os_=500), dict(window=-1), dict(causal=0, window=5),
               dict(sc=float("nan")), dict(sc=float("inf")), dict(nws=0)):
        assert att(ok, **kw) == -2, kw
    assert att(ok, q=None) == -1 and att(ok, out=None) == -1 and att(ok, ws=None) == -1
    assert att(ok, q=0x1008) == -3 and att(ok, out=0x1008) == -3 and att(ok, ws=0x1010) == -3
    assert att(ok, tokens=0, max_q=0, q=None, out=None) == 0  # nothing to do
    app = lambda c, layer=0, tokens=1, dt=0, k=P, ks=256, v=P, vs=256, w=P, st=P: L.tq_kv4_append(
        c, layer, tokens, dt, k, ks, v, vs, w, st, None)
    assert app(None) == -1 and app(ok, layer=2) == -2 and app(ok, ks=255) == -2 and app(ok, dt=5) == -2
    assert app(ok, k=None) == -1 and app(ok, st=None) == -1 and app(ok, k=0x1001) == -3 and app(ok, tokens=0) == 0
    assert L.tq_kv4_read(ok, 0, 1, 0, P, 0x1008, P, P, None) == -3 and L.tq_kv4_read(ok, 0, -1, 0, P, P, P, P, None) == -2
    assert L.tq_kv4_extend(ok, 0, P, P, 1, P, P, P, 1 << 20, P, None) == -2
    assert L.tq_kv4_extend(ok, 1, P, P, 1, P, None, P, 1 << 20, P, None) == -1
    assert L.tq_kv4_extend(ok, 1, P, P, 1, P, P, P, 16, P, None) == -2  # workspace too small
    assert L.tq_kv4_fork(ok, 1, None, P, P, None) == -1 and L.tq_kv4_fork(ok, 0, P, P, P, None) == -2
    assert L.tq_kv4_free(ok, 1, 0x1002, None, P, None) == -3
    assert L.tq_kv4_compact(ok, P, P, P, None, P, 1 << 20, P, None) == -1
    other = cache(tq, layers=3)
    assert L.tq_kv4_copy_pages(ok, other, 1, P, P, P, None) == -2


def test_w4_argument_errors_without_gpu():
    from paper_2609_09240_gb300 import tq
    L = tq.lib()
    assert L.tq_w4_bytes(17, 256) == 2 * 2 * 1088 and L.tq_w4_bytes(16, 100) == 0 and L.tq_w4_bytes(0, 128) == 0
    P = 0x1000
    w = tq.tq_w4_weight(16, 256)
    w.tiles = P
    r = ctypes.byref(w)
    lin = lambda M=1, N=16, K=256, w=r, x=P, y=P, ws=P, n=1 << 30: L.tq_w4_linear(M, N, K, w, x, y, ws, n, None)
    assert lin(M=0) == -2 and lin(N=17) == -2 and lin(K=128) == -2 and lin(K=200) == -2 and lin(n=0) == -2
    assert lin(w=None) == -1 and lin(x=None) == -1 and lin(y=None) == -1 and lin(ws=None) == -1
    assert lin(x=0x1008) == -3 and lin(y=0x1001) == -3 and lin(ws=0x1080) == -3
    assert L.tq_w4_linear_f32out(1, 16, 256, r, P, 0x1002, P, 1 << 30, None) == -3
    assert L.tq_w4_pack(16, 130, P, P, P, P, P, None) == -2 and L.tq_w4_pack(16, 128, None, P, P, P, P, None) == -1
    assert L.tq_w4_quantize(16, 128, 0x1004, P, P, None) == -3 and L.tq_w4_dequantize(16, 256, r, 0x1008, None) == -3
    assert L.tq_w4_workspace_bytes(0, 16, 128) == 0 and L.tq_w4_workspace_bytes(1, 16, 128) > 0
