"""The kernel for many query rows of the attention over the 4-bit K/V cache, in
calls whose sequences are known to reach it: the rule between the two kernels
(csrc/tq_kv4_rule.cuh) is compiled for the host and asked."""
import ctypes
import subprocess

import numpy as np
import pytest

import test_gpu_kv4 as base
import test_gpu_kv4_ranges as ranges
from test_gpu_kv4 import i32, make, run_attention

pytestmark = pytest.mark.gpu

RULE = r"""
#include "tq_kv4_rule.cuh"
using namespace tq::kv4;
extern "C" void route(int count, const int *n, const int *L, int q_heads, int heads, int dim, int window, int *tiles) {
  int64_t tokens = 0;
  uint64_t all = 0;
  int max_q = 0, p0;
  for (int b = 0; b < count; ++b) {
    tokens += n[b], max_q = n[b] > max_q ? n[b] : max_q;
    all += work_of_many(n[b], q_heads, heads, pages_seen(L[b], n[b], window, &p0));
  }
  for (int b = 0; b < count; ++b)
    tiles[b] = call_of_many(tokens, max_q, q_heads, heads, dim) &&
               goes_to_tiles(n[b], q_heads, heads, dim, pages_seen(L[b], n[b], window, &p0), all);
}
"""


@pytest.fixture(scope="module")
def tq():
    from paper_2609_09240_gb300 import tq
    return tq


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    """Which sequences go to the kernel for many rows."""
    from paper_2609_09240_gb300 import build
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cu").write_text(RULE)
    subprocess.run([build.nvcc(), "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-I", build.CSRC, str(d / "rule.cu"),
                    "-o", str(d / "rule.so")], check=True)
    lib = ctypes.CDLL(str(d / "rule.so"))

    def ask(lengths, n, heads, group, D, window=0):
        a, b, out = (np.ascontiguousarray(x, np.int32) for x in (n, lengths, np.zeros(len(n))))
        lib.route(len(n), *(x.ctypes.data_as(ctypes.c_void_p) for x in (a, b)), heads * group, heads, D, window,
                  out.ctypes.data_as(ctypes.c_void_p))
        return out.astype(bool).tolist()
    return ask


def test_the_cases_of_the_other_files_reach_it(route):
    for lengths, n, heads, group, D, window, some in (
            ([333, 130, 257, 40, 63, 200], [150, 130, 1, 33, 7, 2], 4, 8, 128, 0, 4),
            ([333, 130, 257, 40, 63, 200], [150, 130, 1, 33, 7, 2], 8, 4, 64, 90, 3),
            ([2, 0, 100, 5], [200, 2, 0, 260], 2, 8, 128, 0, 2), ([2, 0, 100, 5], [200, 2, 0, 260], 4, 4, 64, 0, 2),
            ([128, 256, 129, 127, 384], [128, 64, 65, 63, 1], 4, 8, 128, 0, 4), ([300], [220], 4, 8, 128, 0, 1),
            ([2, 0, 100, 1], [210, 70, 4, 99], 4, 8, 128, 2 ** 31 - 1, 3), ([300], [200], 4, 8, 128, 0, 1),
            ([400], [210], 4, 8, 128, 0, 1), ([330, 260], [170, 60], 4, 8, 128, 0, 2)):
        assert sum(route(lengths, n, heads, group, D, window)) == some, (lengths, n)


@pytest.mark.parametrize("D,heads,group", [(128, 4, 8), (64, 8, 5)])
@pytest.mark.parametrize("kw", [dict(qscale=12.0), dict(qscale=1e-4), dict(scale=0.0), dict(scale=-0.2), dict(qscale=40.0)])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_sharp_flat_and_falling_scores(tq, route, D, heads, group, kw, dtype):
    lengths, n = [700, 600], [170, 140]
    assert all(route(lengths, n, heads, group, D))
    run_attention(tq, lengths, n, heads, group, D, dtype, seed=24, **kw)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_scores_of_ten_digits_in_heads_of_64(tq, route, dtype):
    assert all(route([400], [230], 4, 8, 64))
    ranges.test_scores_of_ten_digits(tq, dtype, 64, 400, 230, 4, 8)


@pytest.mark.parametrize("D,heads,group", [(128, 2, 8), (64, 4, 6)])
def test_more_prompts_than_the_longest_first_order_sorts(tq, route, D, heads, group):
    lengths, n = [80 + 3 * i for i in range(40)], [25 + (i % 3) * 15 for i in range(40)]
    assert all(route(lengths, n, heads, group, D))
    run_attention(tq, lengths, n, heads, group, D, seed=9)


# ------------------------------------------------------------- mixed batches
def test_few_queries_on_a_long_cache_beside_prompts(tq, route):
    lengths, n = [400, 400, 20000, 70], [200, 200, 12, 1]
    assert route(lengths, n, 4, 8, 128) == [True, True, False, False]
    run_attention(tq, lengths, n, 4, 8, 128, seed=71)


@pytest.mark.parametrize("count", [33, 600])
def test_prompts_among_decoding_sequences(tq, route, count):
    """Over 32 sequences, and over the 512 that a block's threads look at together."""
    lengths = [20 + (11 * i) % 150 for i in range(count)]
    n = [1] * count
    for b in (3, count // 2, count - 5):
        lengths[b], n[b] = 200, 160
    n[7], n[9] = 0, 20
    assert [b for b, t in enumerate(route(lengths, n, 2, 8, 64)) if t] == [3, 9, count // 2, count - 5]
    run_attention(tq, lengths, n, 2, 8, 64, seed=72, max_q=160)


def test_a_batch_of_decoding_sequences_without_max_q(tq, route):
    lengths = [30 + i for i in range(230)]
    assert not any(route(lengths, [1] * 230, 2, 16, 128))
    run_attention(tq, lengths, [1] * 230, 2, 16, 128, seed=73)


# --------------------------------------------- errors, repetition, addresses
def test_bad_lists_are_reported_and_harmless(tq, route):
    import torch
    lengths, n, T = [300, 400, 200], [220, 60, 30], 310
    c, *_ = make(tq, lengths, 2, 128, seed=71)
    assert all(route(lengths, n, 2, 16, 128)) and all(route([300, 200], [220, 30], 2, 16, 128))
    q = torch.randn((T, 32, 128), device="cuda").half()
    out = torch.empty_like(q)
    table, length = c.table.clone(), c.length.clone()
    clean = tq.tq_kv4_attention(q, c, 1, i32([0, 1, 2]), i32([0, 220, 280, 310])).clone()
    c.check()
    for slots, indptr, breakage in (([0, 7, 2], [0, 220, 280, 310], None), ([0, 1, -1], [0, 220, 280, 310], None),
                                    ([0, 1, 2], [0, 220, 500, 310], None), ([0, 1, 2], [0, 220, -3, 310], None),
                                    ([0, 1, 2], [0, 220, 280, 2 ** 31 - 1], None), ([0, 1, 2], [0, 220, 280, 310], "table"),
                                    ([0, 1, 2], [0, 220, 280, 310], "length"), ([0, 1, 2], [0, 220, 280, 310], "negative"),
                                    ([0, 1, 2], [0, 220, 280, 310], "own table")):
        if breakage == "table":
            c.table[1, 2] = 10 ** 6
        if breakage in ("length", "negative"):
            c.length[1] = 10 ** 6 if breakage == "length" else -5
        if breakage == "own table":
            c.table[0, 1], c.table[0, 3] = -7, c.pages
        out.zero_()
        tq.tq_kv4_attention(q, c, 1, i32(slots), i32(indptr), out=out)
        with pytest.raises(tq.TQError):
            c.check()
        if breakage == "own table":
            # a sequence without some of its pages: unspecified, the others are not
            assert torch.equal(out[220:], clean[220:])
        else:
            assert torch.equal(out[:220], clean[:220])
        c.table.copy_(table), c.length.copy_(length)
    assert torch.equal(tq.tq_kv4_attention(q, c, 1, i32([0, 1, 2]), i32([0, 220, 280, 310])), clean)
    c.check()
    assert tq.tq_get_device_status() == 0


@pytest.mark.parametrize("lengths,n,D", [([2000, 300], [250, 3], 128), ([900] * 35, [16] * 34 + [1], 64)])
def test_same_bits_again_and_on_another_stream(tq, route, lengths, n, D):
    import torch
    assert any(route(lengths, n, 2, 16, D))
    c, *_ = make(tq, lengths, 2, D, seed=81)
    q = torch.randn((sum(n), 32, D), device="cuda").half()
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


def test_cache_larger_than_32_bits(tq, route):
    """Pages whose bytes lie past 2^32."""
    import torch
    from oracle import q4
    D, heads, group, L, n = 128, 8, 4, 220, 200
    assert all(route([L], [n], heads, group, D))
    pages = (1 << 32) // (q4.block_bytes(D) * heads) + 40
    data = torch.zeros((1, pages, heads, q4.block_bytes(D)), dtype=torch.uint8, device="cuda")
    held = [pages - 1, 3, pages - 2, pages - 7]
    table = i32(held).reshape(1, 4)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[held] = 1
    c = tq.Kv4Cache(data, table, i32([L]), refs, D)
    k, v = (torch.randn((L, heads, D), device="cuda").half() for _ in "kv")
    pos = np.arange(L)
    where = i32(np.array(held)[pos // 64] * 64 + pos % 64)
    tq.tq_kv4_append(k, v, c, 0, where)
    q = torch.randn((n, heads * group, D), device="cuda").half()
    out = torch.empty_like(q)
    lse = torch.empty((n, heads * group), dtype=torch.float32, device="cuda")
    tq.tq_kv4_attention(q, c, 0, i32([0]), i32([0, n]), out=out, lse=lse)
    c.check()
    near = data[:, held].cpu().numpy()  # the same pages in a small pool
    base.check_attention(c, near, np.arange(4, dtype=np.int32).reshape(1, 4), np.array([L]), [0], [n], heads, group, D, 0, q,
                         out, lse, True, 0, D ** -0.5, "fp16")
    del data, c
    torch.cuda.empty_cache()
