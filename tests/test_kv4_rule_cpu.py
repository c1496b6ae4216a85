"""Which of the two attention kernels over the 4-bit K/V cache a sequence goes to
(csrc/tq_kv4_rule.cuh compiled for the host): the rule's cases, its arithmetic at
the ends of what the calls accept, and that the launched blocks suffice."""
import subprocess

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "tq_kv4_rule.cuh"

using namespace tq::kv4;
struct Seq { int n, L; };

static std::vector<bool> route(const std::vector<Seq> &seqs, int q_heads, int heads, int dim, int window) {
  int64_t tokens = 0;
  int max_q = 0, p0;
  uint64_t all = 0;
  for (auto &s : seqs) {
    tokens += s.n, max_q = std::max(max_q, s.n);
    all += work_of_many(s.n, q_heads, heads, pages_seen(s.L, s.n, window, &p0));
  }
  std::vector<bool> r;
  const bool call = call_of_many(tokens, max_q, q_heads, heads, dim);
  for (auto &s : seqs)
    r.push_back(call && goes_to_tiles(s.n, q_heads, heads, dim, pages_seen(s.L, s.n, window, &p0), all));
  return r;
}
static int failed = 0;
static void want(const char *what, std::vector<bool> got, std::vector<bool> exp) {
  if (got != exp) printf("%s\n", what), failed = 1;
}

int main() {
  using V = std::vector<bool>;
  want("decode", route(std::vector<Seq>(400, Seq{1, 3000}), 32, 8, 128, 0), V(400, false));
  want("one sequence below the rows", route({{187, 6000}}, 32, 8, 128, 0), V{false});
  want("one sequence at the rows", route({{188, 6000}}, 32, 8, 128, 0), V{true});
  want("heads of 64", route({{188, 6000}}, 32, 8, 64, 0), V{false});
  want("heads of 64, more rows", route({{219, 6000}}, 32, 8, 64, 0), V{true});
  want("sixteen sequences", route(std::vector<Seq>(16, Seq{12, 2000}), 32, 8, 128, 0), V(16, true));
  // a few queries on a long cache: not beside decoding sequences, not beside prompts
  std::vector<Seq> mixed(400, Seq{1, 2000});
  mixed.push_back({12, 131072});
  want("few on a long cache beside decoding", route(mixed, 32, 8, 128, 0), V(401, false));
  want("few on a long cache beside prompts", route({{1000, 2000}, {1000, 2000}, {12, 131072}}, 32, 8, 128, 0),
       V{true, true, false});
  // the window, not the cache, is what its queries see
  want("few under a window", route({{1000, 2000}, {1000, 2000}, {12, 131072}}, 32, 8, 128, 1000), V{true, true, true});
  want("under 48 rows a head", route({{1000, 2000}, {11, 2000}, {1, 100}, {0, 50}}, 32, 8, 128, 0), V{true, false, false, false});
  want("no tokens", route({{300, 0}, {300, 5}}, 32, 8, 128, 0), V{true, true});

  // the first position seen, with the widest windows
  int p0;
  for (int64_t L : {0ll, 1ll, 100ll, 1ll << 30})
    for (int64_t n : {1ll, 2ll, 3ll, 101ll, (1ll << 31) - 1})
      for (int64_t w : {0ll, 1ll, 64ll, 1ll << 30, (1ll << 31) - 1}) {
        const int64_t pos = L - n, first = w > 0 ? std::max<int64_t>(0, pos - w + 1) : 0;
        const int np = pages_seen((int)L, (int)n, (int)w, &p0);
        if (first_seen((int)pos, (int)w) != first || p0 != first / 64 || np != (L + 63) / 64 - first / 64)
          printf("window %lld of %lld, %lld\n", (long long)w, (long long)L, (long long)n), failed = 1;
      }
  // sums of the largest calls do not wrap
  if (work_of_many(1 << 17, 1 << 14, 1, 1 << 24) != 1ull << 55) printf("work\n"), failed = 1;

  // the blocks that a call launches
  std::mt19937 rng(1);
  for (int it = 0; it < 20000; ++it) {
    const int g = 1 + rng() % 20, count = 1 + rng() % 40;
    int64_t tokens = 0, tiles = 0;
    for (int b = 0; b < count; ++b) {
      const int n = rng() % (rng() % 3 ? 4 : 700);
      tokens += n;
      if ((int64_t)n * g >= kManyRows) tiles += ((int64_t)n * g + kTileRows - 1) / kTileRows;
    }
    if (tiles > most_row_tiles(tokens, g, count)) printf("blocks\n"), failed = 1;
  }
  // few of them where few can work: one or two rows a sequence
  if (most_row_tiles(200, 4, 200) > 16) printf("blocks of a decode batch\n"), failed = 1;
  return failed;
}
"""


def test_rule(tmp_path):
    from paper_2609_09240_gb300 import build
    (tmp_path / "rule.cu").write_text(PROGRAM)
    exe = str(tmp_path / "rule")
    subprocess.run([build.nvcc(), "-std=c++17", "-I", build.CSRC, str(tmp_path / "rule.cu"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
