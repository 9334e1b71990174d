"""The division of attention over a 4-bit cache (csrc/lg_q4_plan.cuh), compiled for the host: an item's
units against the blocks of its tiles, and the shares of random batches (every block of every item
exactly once, at most one piece in each of a CTA's two slots, and the merge's range of parts)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_10044_gb300", "csrc")

PROG = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "lg_q4_plan.cuh"
using namespace lg;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static std::mt19937_64 rng(11);
static int64_t uni(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }
static int pick(std::initializer_list<int> l) { return l.begin()[uni(0, (int)l.size() - 1)]; }

int main() {
  for (int it = 0; it < 3000; ++it) {
    Q4Shape s;
    s.g = (int)uni(1, 8);
    s.rows = pick({8, 16, 24, 32});
    s.window = uni(0, 1) ? (int)uni(1, pick({3, 200, 5000, 2147483647})) : 0;
    s.sink = pick({0, 1, 4, 64, 129, 1000, 2147483647});
    s.H_kv = (int)uni(1, 4);
    std::vector<ChunkSeq> seqs(uni(1, 40));
    int64_t W = 0;
    for (auto &q : seqs) {
      q.n = (int)uni(0, pick({3, 130, 700, 5000}));
      q.m = (int)uni(0, uni(0, 1) ? 20 : 1);
      if (q.m > q.n) q.m = q.n;
      W += q4_seq_units(q, s);
    }
    const int G = (int)uni(1, pick({1, 7, 60, 400}));
    const int64_t step = plan_max(1, (W + G - 1) / G);
    std::vector<int> slots(2 * G, 0);
    int64_t x = 0;
    for (const auto &q : seqs)
      for (int h = 0; h < s.H_kv; ++h)
        for (int t = 0; t < q4_tiles(q, s); ++t) {
          int used;
          const TileRows r = q4_rows(q, s, t, used);
          CHECK(used >= 1 && used <= s.rows && r.first <= r.last && r.last < q.n);
          // the rows its queries see, by the definition
          const TileBlocks b = tile_blocks(r, kQ4Bn2);
          for (int u = t * s.rows; u < t * s.rows + used; ++u) {
            const int own = q.n - q.m + u / s.g;
            for (int i : {0, own, own - s.window + 1, s.sink - 1, (int)uni(0, own)}) {
              if (i < 0 || i > own) continue;
              if (s.window && i <= (int64_t)own - s.window && i >= s.sink) continue;
              bool in = false;
              for (int k = 0; k < b.count; ++k) in |= b.index(k) == i >> kQ4Bn2;
              CHECK(in);
            }
          }
          const int units = q4_units(q, s);
          CHECK(b.count >= 1 && b.count + kQ4ItemUnits <= units);
          // pieces
          const int c0 = (int)(x / step), c1 = (int)((x + units - 1) / step);
          CHECK(c1 < G);
          int done = 0, pieces = 0;
          for (int c = c0; c <= c1; ++c) {
            const int k0 = q4_cut(c * step - x, b.count), k1 = q4_cut((c + 1) * step - x, b.count);
            CHECK(k0 == done);
            done = k1;
            if (k0 < k1) {
              ++pieces;
              if (!(k0 == 0 && k1 == b.count)) ++slots[2 * c + (x < c * step ? 0 : 1)];
            }
          }
          CHECK(done == b.count);
          // the merge, as the CTA whose start is the first to cut the item sees it
          if (c1 > c0) {
            CHECK(x < (c0 + 1) * step && (c0 + 1) * step - step <= x);
            auto cut = [&](int c) { return q4_cut(c * step - x, b.count); };
            int p0 = 0, p1 = c1 + 1 - c0;
            while (cut(c0 + p0 + 1) == 0) ++p0;
            while (cut(c0 + p1 - 1) == b.count) --p1;
            CHECK(p1 - p0 == pieces);
          } else {
            CHECK(pieces == 1);
          }
          x += units;
        }
    CHECK(x == W);
    for (int v : slots) CHECK(v <= 1);
  }
  puts("ok");
}
"""


def test_division(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROG)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout
