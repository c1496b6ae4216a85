"""The 4-bit K/V cache on the GPU against its definitions in numpy.

Attention's tolerance, per output (float64 reference o, a = sum p |v|, A the
largest scale * sum |q k| that the row sees):
  2^-11 |o| (2^-8 in bf16): the output's rounding;
  2^-11 a: p is rounded to fp16 for its product with v;
  2^-17 (1 + A) a: float32 scores (128 products, relative error of the sum of
    magnitudes below 2^-18), which the exponential turns into a relative
    error of p, its own error and the sum's;
  2^-24: results below fp16's normal range.
Everything the upkeep of pages returns is compared bit for bit.
"""
import numpy as np
import pytest

from oracle import q4

pytestmark = pytest.mark.gpu
PAGE = 64


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def i32(v):
    return dev(np.asarray(v, np.int32).reshape(-1))


def random_blocks(rng, shape, D, mean=0.0):
    """Blocks of valid codes and params; mean shifts what the codes stand for."""
    data = rng.integers(0, 256, shape + (q4.block_bytes(D),)).astype(np.uint8)
    n = shape + (2 * (D // 64) * PAGE,)
    s = np.exp(rng.normal(-1.5, 0.5, n)).astype(np.float16).view(np.uint16) & 0xFFF0
    z = np.clip(np.rint(rng.normal(7.5 - 4 * mean, 1.0, n)), 0, 15).astype(np.uint16)
    data[..., PAGE * D:] = (s | z).view(np.uint8)
    return data


def make(tq, lengths, heads, D, layers=2, spare=3, seed=0, max_pages=None, poison=True):
    """A cache with one sequence per slot in pages at random; what no token
    owns stands for NaN."""
    rng = np.random.default_rng(seed)
    need = [-(-n // PAGE) for n in lengths]
    pages = sum(need) + spare
    data = random_blocks(rng, (layers, pages, heads), D)
    order = rng.permutation(pages)
    W = max_pages or max(need + [1]) + 1
    table = np.full((len(lengths), W), -1, np.int32)
    at, refs = 0, np.zeros(pages, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        refs[table[b, :n]] = 1
        at += n
        if n and poison and lengths[b] % PAGE:
            par = data[:, table[b, n - 1], :, PAGE * D:].copy().view(np.uint16).reshape(layers, heads, -1, PAGE)
            par[..., lengths[b] % PAGE:] = 0x7FF3
            data[:, table[b, n - 1], :, PAGE * D:] = par.reshape(layers, heads, -1).view(np.uint8)
    if poison:
        data[:, order[at:]] = 0xFF
    length = np.asarray(lengths, np.int32)
    return tq.Kv4Cache(dev(data), dev(table), dev(length), dev(refs), D), data, table, length, refs


def run_attention(tq, lengths, n, heads, group, D, dtype="fp16", causal=True, window=0, scale=None, seed=0, slots=None,
                  qscale=1.0, max_q=None, layer=1, pad=0, layers=2):
    import torch
    c, data, table, length, _ = make(tq, lengths, heads, D, seed=seed, layers=layers)
    rng = np.random.default_rng(seed + 1)
    slots = list(range(len(lengths))) if slots is None else slots
    T, Hq = sum(n), heads * group
    dt = {"fp16": torch.float16, "bf16": torch.bfloat16}[dtype]
    q = dev((rng.standard_normal((T, Hq, D)) * qscale).astype(np.float32)).to(dt)
    if pad:  # token rows further apart than the heads are wide
        wide = torch.full((T, Hq * D + pad), float("nan"), dtype=dt, device="cuda")
        wide[:, :Hq * D] = q.flatten(1)
        q = wide[:, :Hq * D].unflatten(1, (Hq, D))
    indptr = i32(np.concatenate([[0], np.cumsum(n)]))
    out = torch.full((T, Hq, D), float("nan"), dtype=dt, device="cuda")
    lse = torch.full((T, Hq), float("nan"), dtype=torch.float32, device="cuda")
    tq.tq_kv4_attention(q, c, layer, i32(slots), indptr, max_q=max_q, scale=scale, causal=causal, window=window, out=out,
                        lse=lse)
    torch.cuda.synchronize()
    c.check()
    return check_attention(c, data, table, length, slots, n, heads, group, D, layer, q, out, lse, causal, window,
                           D ** -0.5 if scale is None else scale, dtype)


def check_attention(c, data, table, length, slots, n, heads, group, D, layer, q, out, lse, causal, window, scale, dtype):
    qf, got, gl = q.float().cpu().numpy().astype(np.float64), out.float().cpu().numpy(), lse.cpu().numpy()
    at = 0
    for b, s in enumerate(slots):
        for h in range(heads):
            K, V = q4.sequence(data, table, length, s, layer, h, D)
            for g in range(group):
                hq = h * group + g
                o, l, a, A = q4.attention(qf[at:at + n[b], hq], K, V, int(length[s]) - n[b], scale, causal, window)
                tol = np.abs(o) * 2.0 ** (-11 if dtype == "fp16" else -8) + (
                    2.0 ** -11 + 2.0 ** -17 * (1 + A[:, None])) * a + 2.0 ** -24
                err = np.abs(got[at:at + n[b], hq] - o)
                assert np.all(err <= tol), (b, hq, float((err / tol).max()), np.argwhere(~(err <= tol))[:3])
                le = gl[at:at + n[b], hq]
                assert np.array_equal(np.isneginf(le), np.isneginf(l))
                f = np.isfinite(l)
                assert np.all(np.abs(le[f] - l[f]) <= 2.0 ** -17 * (1 + A[f]) + 2.0 ** -21 * np.abs(l[f]))
        at += n[b]
    return c


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 8), (3, 5), (1, 17)])
def test_decode_lengths_around_pages(tq, D, dtype, heads, group):
    lengths = [1, 2, 63, 64, 65, 127, 128, 129, 200, 511, 513]
    run_attention(tq, lengths, [1] * len(lengths), heads, group, D, dtype, max_q=1)


@pytest.mark.parametrize("D,group", [(128, 4), (64, 3), (128, 9)])
@pytest.mark.parametrize("window", [0, 1, 63, 64, 100, 1000])
def test_several_queries_and_windows(tq, D, group, window):
    lengths, n = [5, 70, 300, 129, 64, 1], [5, 3, 9, 1, 64, 1]
    run_attention(tq, lengths, n, 2, group, D, window=window, seed=window + 1)


@pytest.mark.parametrize("D,group,dtype", [(128, 4, "fp16"), (64, 2, "fp16"), (128, 1, "bf16"), (128, 7, "fp16")])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 90)])
def test_many_queries(tq, D, group, dtype, causal, window):
    lengths, n = [333, 130, 257, 40], [150, 130, 1, 33]
    run_attention(tq, lengths, n, 2, group, D, dtype, causal=causal, window=window, seed=7)


@pytest.mark.parametrize("D,heads,group,dtype", [(128, 4, 8, "fp16"), (64, 8, 4, "fp16"), (128, 8, 5, "bf16"),
                                                 (64, 2, 19, "bf16"), (128, 32, 1, "fp16")])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 90)])
def test_enough_rows_for_the_tile_kernel(tq, D, heads, group, dtype, causal, window):
    """Over 6000 query rows: prompts go to the kernel that decodes whole tiles,
    the single queries and the few among them do not."""
    lengths, n = [333, 130, 257, 40, 63, 200], [150, 130, 1, 33, 7, 2]
    run_attention(tq, lengths, n, heads, group, D, dtype, causal=causal, window=window, seed=17)


def test_tile_kernel_edges(tq):
    # positions below zero, empty sequences and ranges, lengths around tiles of 128
    run_attention(tq, [2, 0, 100, 5], [200, 2, 0, 260], 2, 8, 128, seed=3)
    run_attention(tq, [2, 0, 100, 5], [200, 2, 0, 260], 4, 4, 64, seed=4, causal=False)
    run_attention(tq, [128, 256, 129, 127, 384], [128, 64, 65, 63, 1], 4, 8, 128, seed=5)
    run_attention(tq, [2000, 700], [60, 150], 4, 8, 128, seed=6, window=257)
    # sharp, flat, growing and shrinking scores
    for i, kw in enumerate((dict(qscale=12.0), dict(qscale=1e-4), dict(scale=0.0), dict(scale=-0.2), dict(qscale=40.0))):
        run_attention(tq, [700, 300], [100, 140], 4, 8, 128, seed=24 + i, **kw)
    run_attention(tq, [100, 200, 300], [60, 190], 4, 8, 128, slots=[1, 1], pad=8, seed=33)


def test_more_prompts_than_the_longest_first_order_sorts(tq):
    # over 32 sequences the blocks go sequence by sequence
    lengths = [50 + 3 * i for i in range(40)]
    run_attention(tq, lengths, [20 + (i % 3) * 15 for i in range(40)], 2, 4, 64, seed=9)


def test_tile_kernel_keeps_what_is_not_a_number_to_its_rows(tq):
    """As below for the kernel of few rows; here the row's own position also
    decides whether it sees the token that stands for NaN."""
    import torch
    D, heads, group = 128, 4, 8
    n, L = 220, 300
    for value in (False, True):
        c, data, table, length, refs = make(tq, [L], heads, D, seed=62)
        at = PAGE * D + (2 * PAGE * 2 if value else 0) + 2 * (1 * PAGE + 200 % PAGE)  # group 1 of token 200, head 1
        data[1, table[0, 200 // PAGE], 1, at], data[1, table[0, 200 // PAGE], 1, at + 1] = 0xF0, 0x7F
        q = dev(np.random.default_rng(1).standard_normal((n, heads * group, D)).astype(np.float16))
        q[5, 3, 0] = float("nan")
        args = (c, 1, i32([0]), i32([0, n]))
        clean = tq.tq_kv4_attention(q, *args).float().cpu().numpy()
        c.data.copy_(dev(data))
        out = tq.tq_kv4_attention(q, *args).float().cpu().numpy()
        bad = np.zeros(out.shape, bool)
        bad[200 - (L - n):, group:2 * group, 64 if value else 0:] = True  # rows from position 200 on
        bad[5, 3] = True
        assert np.isnan(out[bad]).all()
        assert np.isfinite(out[~bad]).all() and np.array_equal(out[~bad], clean[~bad])


def test_more_queries_than_tokens_and_empty_sequences(tq):
    # positions below zero see nothing: zeros and lse -inf; an empty sequence
    # and an empty range are fine anywhere in the list
    for n in ([3, 2, 0, 7], [200, 2, 0, 260]):
        run_attention(tq, [2, 0, 100, 5], n, 2, 4, 128, seed=3)
        run_attention(tq, [2, 0, 100, 5], n, 1, 2, 64, seed=4, causal=False)


def test_long_sequences_split_over_the_chip(tq):
    run_attention(tq, [20000], [1], 2, 4, 128, seed=11, max_q=1)
    run_attention(tq, [9000, 100, 17011], [1, 1, 2], 1, 6, 64, seed=12, max_q=2)
    run_attention(tq, [7000], [40], 1, 4, 128, seed=13)


def test_sharp_and_flat_softmax(tq):
    run_attention(tq, [700, 64], [2, 1], 2, 4, 128, qscale=12.0, seed=21)
    run_attention(tq, [700, 64], [2, 1], 2, 4, 128, qscale=1e-4, seed=22)
    run_attention(tq, [700, 64], [2, 1], 2, 4, 128, scale=0.0, seed=23)
    run_attention(tq, [700, 300], [2, 140], 2, 4, 128, scale=-0.2, seed=24)
    run_attention(tq, [500, 300], [2, 140], 1, 4, 128, qscale=30.0, seed=25)


def test_rows_apart_slots_out_of_order_and_repeated_reads(tq):
    run_attention(tq, [100, 200, 300], [1, 1, 1], 2, 4, 128, slots=[2, 0, 1], pad=24, seed=31)
    run_attention(tq, [100, 200, 300], [1, 1], 2, 4, 64, slots=[1, 1], pad=8, seed=32)
    run_attention(tq, [100, 200, 300], [40, 90], 2, 4, 128, slots=[1, 1], pad=8, seed=33)


def test_more_sequences_than_a_launch_takes(tq):
    # lists are worked through 512 sequences at a time
    lengths = [(7 * i) % 150 for i in range(1030)]
    run_attention(tq, lengths, [1 if i % 9 else 0 for i in range(1030)], 1, 2, 64, seed=43, max_q=1)
    lengths = [20 + (7 * i) % 100 for i in range(530)]
    run_attention(tq, lengths, [20 if i in (3, 520) else 1 for i in range(530)], 2, 8, 64, seed=44, max_q=20)


def test_small_max_q_costs_no_results(tq):
    run_attention(tq, [400, 90], [150, 1], 2, 4, 128, max_q=1, seed=41)


def test_extreme_scales_of_values(tq):
    """Values from fp16's smallest scales to its largest, keys ordinary."""
    import torch
    c, data, table, length, refs = make(tq, [500, 70], 2, 128, seed=51)
    rng = np.random.default_rng(52)
    par = data[..., PAGE * 128 + 2 * PAGE * 2:].copy().view(np.uint16)  # V params
    nan = (par & 0x7FF0) > 0x7C00
    e = np.exp2(rng.uniform(-20, 12, par.shape)).astype(np.float16).view(np.uint16) & 0xFFF0
    par = np.where(nan, par, e | (par & 15)).astype(np.uint16)
    data[..., PAGE * 128 + 2 * PAGE * 2:] = par.view(np.uint8)
    c.data.copy_(dev(data))
    n = [3, 1]
    q = dev(rng.standard_normal((4, 8, 128)).astype(np.float16))
    lse = torch.empty((4, 8), dtype=torch.float32, device="cuda")
    out = tq.tq_kv4_attention(q, c, 0, i32([0, 1]), i32([0, 3, 4]), lse=lse)
    check_attention(c, data, table, length, [0, 1], n, 2, 4, 128, 0, q, out, lse, True, 0, 128 ** -0.5, "fp16")


def test_what_is_not_a_number_stays_in_its_rows(tq):
    """A query that holds an infinity or a NaN, and a cached group that stands
    for NaN, spoil the outputs that depend on them and no others."""
    import torch
    for n0 in (1, 60):
        c, data, table, length, refs = make(tq, [300, 200], 2, 128, seed=61)
        data[1, table[1, 1], 1, PAGE * 128 + 2 * (0 * PAGE + 9)] = 0xF0  # slot 1, head 1: K param of token 73
        data[1, table[1, 1], 1, PAGE * 128 + 2 * (0 * PAGE + 9) + 1] = 0x7F
        c.data.copy_(dev(data))
        T = n0 + 1
        q = dev(np.random.default_rng(1).standard_normal((T, 8, 128)).astype(np.float16))
        clean = tq.tq_kv4_attention(q, c, 1, i32([0, 1]), i32([0, n0, T])).float().cpu().numpy()
        q[0, 2, 5], q[0, 3, 7] = float("inf"), float("nan")
        out = tq.tq_kv4_attention(q, c, 1, i32([0, 1]), i32([0, n0, T])).float().cpu().numpy()
        torch.cuda.synchronize()
        bad = np.zeros((T, 8), bool)
        bad[0, 3] = True
        bad[T - 1, 4:] = True  # head 1 of slot 1
        assert np.isnan(out[bad]).all()
        assert not np.isfinite(out[0, 2]).any()
        bad[0, 2] = True
        assert np.isfinite(out[~bad]).all() and np.array_equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("group_of_dims", [0, 1])
def test_values_that_stand_for_nan_spoil_their_dimensions(tq, group_of_dims):
    """Few rows: a NaN group among the values, seen by some of the queries only."""
    D, heads = 128, 2
    for n, window in ((1, 0), (3, 0), (6, 100)):
        c, data, table, length, refs = make(tq, [300], heads, D, seed=63)
        for tok in (120, 298):
            at = PAGE * D + 2 * PAGE * 2 + 2 * (group_of_dims * PAGE + tok % PAGE)
            data[1, table[0, tok // PAGE], 1, at], data[1, table[0, tok // PAGE], 1, at + 1] = 0xF5, 0x7F
        q = dev(np.random.default_rng(1).standard_normal((n, 8, D)).astype(np.float16))
        args = dict(max_q=n, window=window)
        clean = tq.tq_kv4_attention(q, c, 1, i32([0]), i32([0, n]), **args).float().cpu().numpy()
        c.data.copy_(dev(data))
        out = tq.tq_kv4_attention(q, c, 1, i32([0]), i32([0, n]), **args).float().cpu().numpy()
        bad = np.zeros(out.shape, bool)
        for i in range(n):
            pos = 300 - n + i
            if pos >= 298 or not window:  # 298 in sight, or 120 (never inside the window)
                bad[i, 4:, 64 * group_of_dims:64 * group_of_dims + 64] = True
        assert np.isnan(out[bad]).all()
        assert np.isfinite(out[~bad]).all() and np.array_equal(out[~bad], clean[~bad])


def test_bad_lists_are_reported_and_harmless(tq):
    import torch
    for T0 in (1, 80):
        c, *_ = make(tq, [100, 200], 2, 128, seed=71)
        q = torch.randn((T0 + 1, 8, 128), device="cuda").half()
        for slots, indptr, breakage in (([0, 7], [0, T0, T0 + 1], None), ([-1, 1], [0, T0, T0 + 1], None),
                                        ([0, 1], [0, T0 + 50, T0 + 1], None), ([0, 1], [-3, T0, 1000], None),
                                        ([0, 1], [0, T0, T0 + 1], "table"), ([0, 1], [0, T0, T0 + 1], "length")):
            if breakage == "table":
                c.table[0, 0] = 10 ** 6
            if breakage == "length":
                c.length[1] = 10 ** 6
            tq.tq_kv4_attention(q, c, 1, i32(slots), i32(indptr))
            torch.cuda.synchronize()
            with pytest.raises(tq.TQError):
                c.check()
            c.table[0, 0] = 0


def test_same_bits_again_and_on_another_stream(tq):
    import torch
    for lengths, n in (([5000, 300, 64], [1, 1, 1]), ([2000, 300], [100, 3])):
        c, *_ = make(tq, lengths, 2, 128, seed=81)
        q = torch.randn((sum(n), 8, 128), device="cuda").half()
        args = (c, 1, i32(range(len(n))), i32(np.concatenate([[0], np.cumsum(n)])))
        ref = tq.tq_kv4_attention(q, *args)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        outs = [torch.empty_like(ref) for _ in range(4)]
        for i, o in enumerate(outs):
            tq.tq_kv4_attention(q, *args, out=o, stream=side if i % 2 else None)
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, ref)


def test_graph_of_a_step(tq):
    """extend, append and attend captured once and replayed: each replay adds a
    token, reading lengths and tables on the device."""
    import torch
    D, heads = 128, 2
    c = tq.Kv4Cache.empty(1, 12, heads, D, 3, 4)
    slots, ones = i32([2, 0]), i32([1, 1])
    k = torch.zeros((2, heads, D), device="cuda", dtype=torch.float16)
    v, q = torch.zeros_like(k), torch.zeros((2, 8, D), device="cuda", dtype=torch.float16)
    out = torch.empty_like(q)
    indptr, where = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")

    def step():
        tq.tq_kv4_extend(c, slots, ones, 2, indptr=indptr, where=where)
        tq.tq_kv4_append(k, v, c, 0, where)
        tq.tq_kv4_attention(q, c, 0, slots, indptr, max_q=1, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        tq.tq_kv4_free(c, slots)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = np.random.default_rng(4)
    ks, vs = [], []
    for t in range(70):
        kn, vn, qn = (rng.standard_normal(x.shape).astype(np.float16) for x in (k, v, q))
        k.copy_(dev(kn)), v.copy_(dev(vn)), q.copy_(dev(qn))
        g.replay()
        ks.append(kn), vs.append(vn)
    torch.cuda.synchronize()
    c.check()
    assert c.length.cpu().tolist() == [70, 0, 70]
    got = out.float().cpu().numpy()
    for b in range(2):
        for h in range(heads):
            K, V = (np.stack([np.concatenate([q4.decode(*q4.encode(x[b, h, i:i + 64].astype(np.float32)))
                                              for i in (0, 64)]) for x in xs]) for xs in (ks, vs))
            for j in range(4):
                o, _, a, A = q4.attention(qn[b, 4 * h + j][None].astype(np.float64), K, V, 69, D ** -0.5)
                tol = 2.0 ** -11 * np.abs(o) + (2.0 ** -11 + 2.0 ** -17 * (1 + A[:, None])) * a + 2.0 ** -24
                assert np.all(np.abs(got[b, 4 * h + j] - o) <= tol)


def test_cache_larger_than_32_bits(tq):
    """Pages whose bytes lie past 2^32: offsets are 64 bits throughout."""
    import torch
    D, heads = 128, 8
    pages = (1 << 32) // (q4.block_bytes(D) * heads) + 40
    data = torch.zeros((1, pages, heads, q4.block_bytes(D)), dtype=torch.uint8, device="cuda")
    table = i32([pages - 1, 3, pages - 2]).reshape(1, 3)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[[pages - 1, 3, pages - 2]] = 1
    c = tq.Kv4Cache(data, table, i32([150]), refs, D)
    k, v = (torch.randn((150, heads, D), device="cuda").half() for _ in "kv")
    pos = np.arange(150)
    where = i32(table.cpu().numpy()[0][pos // 64] * 64 + pos % 64)
    tq.tq_kv4_append(k, v, c, 0, where)
    K, V = tq.tq_kv4_read(c, 0, where)
    q = torch.randn((140, 32, D), device="cuda").half()
    for n in (1, 140):
        out = tq.tq_kv4_attention(q[:n], c, 0, i32([0]), i32([0, n])).float()
        a = torch.einsum("nhgd,lhd->nhgl", q[:n].double().unflatten(1, (8, 4)), K.double()) * D ** -0.5
        hidden = torch.arange(150, device="cuda") > torch.arange(150 - n, 150, device="cuda")[:, None]
        p = torch.softmax(a.masked_fill(hidden[:, None, None], -float("inf")), -1)
        o = torch.einsum("nhgl,lhd->nhgd", p, V.double()).flatten(1, 2)
        w = torch.einsum("nhgl,lhd->nhgd", p, V.double().abs()).flatten(1, 2)
        A = D ** -0.5 * torch.einsum("nhgd,lhd->nhgl", q[:n].double().abs().unflatten(1, (8, 4)), K.double().abs())
        tol = 2.0 ** -11 * o.abs() + (2.0 ** -11 + 2.0 ** -17 * (1 + float(A.max()))) * w + 2.0 ** -24
        assert bool(((out - o).abs() <= tol).all())
    c.check()
    del data, c
    torch.cuda.empty_cache()


# ------------------------------------------------------------ append / read
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("layout", ["own", "fused", "odd"])
def test_append_writes_the_definition_and_nothing_else(tq, D, dtype, layout):
    import torch
    heads, T = 3, 70
    dt = {"fp16": torch.float16, "bf16": torch.bfloat16}[dtype]
    c, data, table, length, refs = make(tq, [100, 64, 200], heads, D, seed=5)
    rng = np.random.default_rng(6)
    x = rng.standard_normal((2, T, heads, D)).astype(np.float32)
    x *= np.exp(rng.normal(0, 2, (2, T, heads, 1)))
    x[0, 1, 0], x[1, 2, 1] = 0.0, np.abs(x[1, 2, 1]) + 9
    x[0, 3, 2, 5], x[1, 4, 0, 63], x[0, 5, 1, D - 1] = np.inf, np.nan, -60000
    x[0, 6] *= 1e-6
    kv = [dev(a).to(dt) for a in x]
    if layout != "own":
        step = heads * D + (24 if layout == "fused" else 5)
        wide = [torch.full((T, step), 3.0, dtype=dt, device="cuda") for _ in "kv"]
        off = 8 if layout == "fused" else 1
        for w, t in zip(wide, kv):
            w[:, off:off + heads * D] = t.flatten(1)
        kv = [w[:, off:off + heads * D].unflatten(1, (heads, D)) for w in wide]
    order = rng.permutation(sum(map(int, length)))[:T]
    places = np.concatenate([table[b][np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE for b, n in enumerate(length)])
    where = places[order].astype(np.int32)
    where[10] = -1
    tq.tq_kv4_append(kv[0], kv[1], c, 1, i32(where))
    K, V = tq.tq_kv4_read(c, 1, i32(where), dtype=dt)
    torch.cuda.synchronize()
    c.check()
    want = data.copy()
    kn, vn = (t.float().cpu().numpy() for t in kv)
    for t in range(T):
        if where[t] >= 0:
            for h in range(heads):
                q4.store(want[1, where[t] // PAGE, h], D, where[t] % PAGE, kn[t, h], vn[t, h])
    assert np.array_equal(c.data.cpu().numpy(), want)
    for got, i in ((K, 0), (V, 1)):
        ref = np.stack([np.stack([q4.block_values(want[1, w // PAGE, h], D)[i][w % PAGE] if w >= 0 else np.zeros(D)
                                  for h in range(heads)]) for w in where])
        assert torch.equal(torch.nan_to_num(got, nan=12345.0), torch.nan_to_num(dev(ref).to(dt), nan=12345.0))


def test_append_reports_places_beyond_the_pool(tq):
    import torch
    c, data, *_ = make(tq, [100], 2, 128, seed=5)
    k = torch.ones((2, 2, 128), device="cuda").half()
    for call in (lambda: tq.tq_kv4_append(k, k, c, 0, i32([-5, c.pages * 64])),
                 lambda: tq.tq_kv4_read(c, 0, i32([-5, c.pages * 64]))):
        call()
        with pytest.raises(tq.TQError):
            c.check()
    assert np.array_equal(c.data.cpu().numpy(), data)


def test_binding_refuses(tq):
    import torch
    c, *_ = make(tq, [100], 2, 128)
    q, k = torch.zeros((1, 8, 128), device="cuda").half(), torch.zeros((1, 2, 128), device="cuda").half()
    one, ip = i32([0]), i32([0, 1])
    bad = [lambda: tq.tq_kv4_attention(q.float(), c, 0, one, ip), lambda: tq.tq_kv4_attention(q.cpu(), c, 0, one, ip),
           lambda: tq.tq_kv4_attention(q, c, 0, one, i32([0, 1, 1])), lambda: tq.tq_kv4_attention(q, c, 0, one.long(), ip),
           lambda: tq.tq_kv4_attention(torch.zeros((1, 8, 64), device="cuda").half(), c, 0, one, ip),
           lambda: tq.tq_kv4_attention(q, c, 0, one, ip, lse=torch.zeros((1, 8), device="cuda").half()),
           lambda: tq.tq_kv4_append(k, k.bfloat16(), c, 0, one), lambda: tq.tq_kv4_append(k, k, c, 0, i32([0, 1])),
           lambda: tq.tq_kv4_append(k.transpose(1, 2), k, c, 0, one), lambda: tq.tq_kv4_read(c, 0, one, dtype=torch.float32),
           lambda: tq.Kv4Cache(c.data, c.table, c.length.long(), c.refs, 128)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: tq.tq_kv4_attention(q, c, 2, one, ip), lambda: tq.tq_kv4_attention(q[:, :3], c, 0, one, ip),
              lambda: tq.tq_kv4_attention(q, c, 0, one, ip, window=-1), lambda: tq.Kv4Cache.empty(1, 4, 1, 96, 1, 1),
              lambda: tq.tq_kv4_attention(torch.zeros((2, 8 * 128 + 4), device="cuda").half()[:, :1024].unflatten(
                  1, (8, 128)), c, 0, one, i32([0, 2]))):
        with pytest.raises(tq.TQError):
            f()


# -------------------------------------------------------------------- pages
def same_state(c, ref):
    assert np.array_equal(c.length.cpu().numpy(), ref.length)
    assert np.array_equal(c.refs.cpu().numpy(), ref.refs)
    t = c.table.cpu().numpy()
    for s in range(len(ref.length)):
        n = -(-int(ref.length[s]) // PAGE)
        assert np.array_equal(t[s, :n], ref.table[s, :n]), s


@pytest.mark.parametrize("seed,slots,pages,heads,D,layers", [(0, 6, 40, 2, 64, 3), (1, 40, 500, 1, 128, 2), (2, 3, 7, 1, 64, 1),
                                                             (3, 1500, 20000, 1, 64, 1)])
def test_upkeep_against_the_rules(tq, seed, slots, pages, heads, D, layers):
    """A random life of a cache: extend, fork, free, cut, compact; tables,
    counts, lengths, places and the pool's bytes after every call."""
    import torch
    rng = np.random.default_rng(seed)
    W = 8
    data = rng.integers(0, 256, (layers, pages, heads, q4.block_bytes(D))).astype(np.uint8)
    c = tq.Kv4Cache(dev(data), torch.full((slots, W), -1, dtype=torch.int32, device="cuda"),
                    torch.zeros(slots, dtype=torch.int32, device="cuda"),
                    torch.zeros(pages, dtype=torch.int32, device="cuda"), D)
    ref = q4.Pages(*(x.cpu().numpy() for x in (c.table, c.length, c.refs)))
    refused = 0
    for step in range(40):
        op = rng.choice(["extend", "extend", "extend", "fork", "free", "cut", "compact"])
        some = rng.permutation(slots)[:rng.integers(1, slots + 1)]
        if op == "extend":
            counts = rng.integers(0, rng.choice([2, 70, 200]), len(some))
            got = ref.extend(list(map(int, some)), list(map(int, counts)))
            ip, wh = tq.tq_kv4_extend(c, i32(some), i32(counts), int(counts.sum()))
            if got is None:
                refused += 1
                assert int(c.status.item()) in (64, 128)
                c.status.zero_()
                assert not ip.any().item() and bool((wh == -1).all())
            else:
                assert np.array_equal(ip.cpu().numpy(), got[0]) and np.array_equal(wh.cpu().numpy(), got[1])
                for a, b in ref.copies:
                    data[:, b] = data[:, a]
        elif op == "fork":
            empty = [s for s in range(slots) if ref.length[s] == 0]
            full = [s for s in range(slots) if ref.length[s]]
            if not empty or not full:
                continue
            dst = empty[:rng.integers(1, len(empty) + 1)]
            src = [int(rng.choice(full)) for _ in dst]
            ref.fork(src, dst)
            tq.tq_kv4_fork(c, i32(src), i32(dst))
        elif op in ("free", "cut"):
            keep = None if op == "free" else [int(x) for x in rng.integers(0, 400, len(some))]
            some = some[:max(1, len(some) // 3)]
            keep = keep[:len(some)] if keep else None
            ref.free(list(map(int, some)), keep)
            tq.tq_kv4_free(c, i32(some), None if keep is None else i32(keep))
        else:
            table, refs, remap, n = ref.compact()
            if rng.random() < 0.5:
                to, ro = torch.empty_like(c.table), torch.empty_like(c.refs)
                rm, lv = tq.tq_kv4_compact(c, table_out=to, refs_out=ro)
                same_state(c, ref)
                c.table.copy_(to), c.refs.copy_(ro)
            else:
                rm, lv = tq.tq_kv4_compact(c)
            assert np.array_equal(rm.cpu().numpy(), remap) and int(lv.item()) == n
            assert np.array_equal(c.table.cpu().numpy(), table)
            ref.table, ref.refs = table, refs
            for a, b in ref.copies:
                data[:, b] = data[:, a]
        torch.cuda.synchronize()
        c.check()
        same_state(c, ref)
        assert np.array_equal(c.data.cpu().numpy(), data), (step, op)
    assert refused or seed not in (2,)


def test_upkeep_refuses_bad_lists(tq):
    import torch
    c, data, table, length, refs = make(tq, [100, 0, 70, 0], 1, 64, max_pages=4, spare=2)
    before = [x.clone() for x in (c.data, c.table, c.length, c.refs)]

    def unchanged():
        torch.cuda.synchronize()
        return all(torch.equal(a, b) for a, b in zip(before, (c.data, c.table, c.length, c.refs)))
    for slots, counts, tokens, bit in (([0, 0], [1, 1], 2, 128), ([0, 4], [1, 1], 2, 128), ([-1, 0], [1, 1], 2, 128),
                                       ([0, 1], [1, -1], 0, 128), ([0, 1], [1, 1], 3, 128), ([0, 1], [2, 2], 3, 128),
                                       ([0], [200], 200, 128), ([1, 3], [120, 120], 240, 64), ([1], [2 ** 31 - 1], 5, 128)):
        ip, wh = tq.tq_kv4_extend(c, i32(slots), i32(counts), tokens)
        assert int(c.status.item()) == bit, (slots, counts)
        c.status.zero_()
        assert unchanged() and not ip.any().item() and bool((wh == -1).all())
    for src, dst in (([0], [2]), ([0], [0]), ([0, 0], [1, 1]), ([0, 1], [1, 3]), ([5], [1]), ([0], [-2])):
        tq.tq_kv4_fork(c, i32(src), i32(dst))
        assert int(c.status.item()) == 128
        c.status.zero_()
        assert unchanged(), (src, dst)
    for slots, keep in (([0, 0], None), ([4], None), ([0], [-1])):
        tq.tq_kv4_free(c, i32(slots), None if keep is None else i32(keep))
        assert int(c.status.item()) == 128
        c.status.zero_()
        assert unchanged()
    tq.tq_kv4_free(c, i32([0]), i32([5000]))  # longer than the sequence: nothing to do
    c.check()
    assert unchanged()
    tq.tq_kv4_copy_pages(c, c, i32([0, 99]), i32([-1, 1]))
    assert int(c.status.item()) == 128 and unchanged()
    c.status.zero_()


def test_copy_pages_between_caches(tq):
    import torch
    a, da, *_ = make(tq, [300, 200], 2, 128, seed=1, layers=3)
    b, db, *_ = make(tq, [500], 2, 128, seed=2, layers=3)
    src, dst = [0, 5, 2], [3, 1, 7]
    tq.tq_kv4_copy_pages(a, b, i32(src), i32(dst))
    db[:, dst] = da[:, src]
    assert np.array_equal(b.data.cpu().numpy(), db) and np.array_equal(a.data.cpu().numpy(), da)
    b.check()
    torch.cuda.synchronize()


def test_fork_then_write_leaves_the_parent_alone(tq):
    """Copy on write end to end: children diverge, the parent's answers stay."""
    import torch
    D, heads = 128, 2
    c = tq.Kv4Cache.empty(2, 30, heads, D, 5, 6)
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda n: torch.randn((n, heads, D), generator=g, device="cuda").half()
    ip, wh = tq.tq_kv4_extend(c, i32([0]), i32([100]), 100)
    for layer in range(2):
        tq.tq_kv4_append(rnd(100), rnd(100), c, layer, wh)
    q = torch.randn((1, 8, D), generator=g, device="cuda").half()
    before = [tq.tq_kv4_attention(q, c, layer, i32([0]), i32([0, 1])) for layer in range(2)]
    tq.tq_kv4_fork(c, i32([0, 0, 0]), i32([1, 2, 3]))
    assert c.refs.cpu().tolist()[:3] == [4, 4, 0]
    ip, wh = tq.tq_kv4_extend(c, i32([1, 2, 3]), i32([1, 1, 40]), 42)
    assert c.refs.cpu().tolist()[:6] == [4, 1, 1, 1, 1, 1]
    for layer in range(2):
        tq.tq_kv4_append(rnd(42), rnd(42), c, layer, wh)
    for layer in range(2):
        assert torch.equal(tq.tq_kv4_attention(q, c, layer, i32([0]), i32([0, 1])), before[layer])
    tq.tq_kv4_free(c, i32([1, 2, 3]))
    tq.tq_kv4_free(c, i32([0]))
    c.check()
    assert not c.refs.any().item() and not c.length.any().item() and bool((c.table == -1).all())
