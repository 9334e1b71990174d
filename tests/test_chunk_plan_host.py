"""The division of lg_chunk_attend's work (csrc/lg_chunk_plan.cuh), compiled for the host: the
closed-form costs against their sums, the pieces of random batches (every
key block of every item exactly once, and never more pieces than the two slots of a CTA), and the
blocks against the rows that a tile's queries see."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_10044_gb300", "csrc")

PROG = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <vector>
#include "lg_chunk_plan.cuh"
using namespace lg;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static std::mt19937_64 rng(7);
static int64_t uni(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }
static int pick(std::initializer_list<int> l) { return l.begin()[uni(0, (int)l.size() - 1)]; }

static ChunkShape shape() {
  ChunkShape s;
  s.tok = (int)uni(1, 256);
  s.bn2 = pick({6, 7});
  s.window = uni(0, 2) ? (int)uni(1, pick({3, 200, 5000, 2147483647})) : 0;
  s.sink = pick({0, 1, 4, 64, 129, 1000});
  s.lanes2 = pick({0, 0, 1, 3});
  return s;
}
static ChunkSeq seq() {
  ChunkSeq q;
  q.n = (int)uni(0, pick({3, 130, 700, 5000}));
  q.m = (int)uni(0, uni(0, 1) ? q.n : (q.n < 3 ? q.n : 3));
  return q;
}

int main() {
  for (int it = 0; it < 4000; ++it) {  // costs, tiles, blocks
    const ChunkShape s = shape();
    const ChunkSeq q = seq();
    const int tiles = q.tiles(s.tok), lanes = 1 << s.lanes2;
    int seen = 0;
    for (int r = 0; r < lanes; ++r) {  // the tiles of a line, r, r + lanes, ..
      int64_t sum = 0;
      int k = 0;
      for (int t = r; t < tiles; t += lanes, ++k, ++seen) {
        CHECK(tiles_cost(q, s, r, k) == sum);
        const int64_t c = tile_cost(q, s, t);
        CHECK(c > kItemCost);
        sum += c;
      }
      CHECK(lane_tiles(q, s, r) == k && tiles_cost(q, s, r, k) == sum);
    }
    CHECK(seen == tiles);
    for (int t = 0; t < tiles; ++t) {
      const TileRows r = tile_rows(q, s, t);
      const TileBlocks b = tile_blocks(r, s.bn2);
      // seen by some query of the tile <=> in a block of the tile, up to whole blocks
      std::set<int> want, got;
      for (int j = t * s.tok; j < q.m && j < (t + 1) * s.tok; ++j) {
        const int row = q.n - q.m + j;
        for (int i = 0; i <= row; ++i)
          if (s.window == 0 || (int64_t)i > (int64_t)row - s.window || i < s.sink) want.insert(i >> s.bn2);
      }
      for (int i = 0; i < b.count; ++i) CHECK(got.insert(b.index(i)).second);
      CHECK(want == got);
      // an open block hides no row of its own from any query; others do, or hold sinks
      int o0, o1;
      open_blocks(r, s, b, o0, o1);
      CHECK(o0 >= 0 && o1 >= o0);
      for (int i = 0; i < b.count; ++i) {
        const int64_t i0 = (int64_t)b.index(i) << s.bn2, i1 = i0 + ((int64_t)1 << s.bn2) - 1;
        bool hides = i1 > r.first;
        if (s.window)
          for (int64_t x = i0; x <= i1 && x <= (int64_t)r.last - s.window; ++x) hides |= x >= s.sink;
        if (i >= o0 && i < o1) CHECK(!hides);
        else CHECK(hides || i0 < s.sink);
      }
    }
  }
  for (int it = 0; it < 1500; ++it) {  // pieces
    const ChunkShape s = shape();
    const int lanes = 1 << s.lanes2;
    const int B = (int)uni(1, 12), H = lanes * (int)uni(1, 3), G = pick({1, 2, 19, 152, 304});
    const int lane = (int)uni(0, lanes - 1);  // one line
    std::vector<ChunkSeq> q(B);
    int64_t W = 0, all = 0;
    std::vector<int64_t> start, cost;
    std::vector<int> count;
    for (int b = 0; b < B; ++b) {
      const ChunkSeq x = q[b] = seq();
      all += H / lanes * head_cost(x, s);
      for (int h = 0; h < H; ++h) {
        const int r = first_tile(s, lane, h);
        CHECK(r >= 0 && r < lanes && (r + h) % lanes == lane);
        for (int t = r; t < x.tiles(s.tok); t += lanes) {
          start.push_back(W);
          cost.push_back(tile_cost(x, s, t));
          count.push_back(tile_blocks(tile_rows(x, s, t), s.bn2).count);
          W += cost.back();
        }
      }
    }
    CHECK(all == W);  // every line is as long
    int64_t end = 0;
    const int64_t step = range_step(W, G, s.bn2);
    std::vector<int> next(start.size(), 0);
    for (int c = 0; c < G; ++c) {
      const int64_t y0 = plan_min(W, c * step), y1 = plan_min(W, y0 + step);
      CHECK(y0 == end && y1 >= y0);
      end = y1;
      int slots[2] = {0, 0};
      for (size_t i = 0; i < start.size(); ++i) {
        if (start[i] + cost[i] <= y0 || start[i] >= y1) continue;
        const int b0 = cut_block(y0 - start[i], cost[i], count[i], s.bn2);
        const int b1 = cut_block(y1 - start[i], cost[i], count[i], s.bn2);
        CHECK(b0 == next[i] && b1 >= b0);
        next[i] = b1;
        if (b0 == b1 || (b0 == 0 && b1 == count[i])) continue;
        ++slots[start[i] < y0 ? 0 : 1];
      }
      CHECK(slots[0] <= 1 && slots[1] <= 1);
    }
    CHECK(end == W && (step == 1 << s.bn2 || step * G - W < G));
    for (size_t i = 0; i < start.size(); ++i) CHECK(next[i] == count[i]);
  }
  // the largest line: no 64-bit overflow in the bounds or the cuts
  const ChunkSeq big{2147483647, 2147483647};
  const ChunkShape s{16, 6, 0, 0, 0};
  const int64_t W = tiles_cost(big, s, 0, big.tiles(s.tok)) / 2;
  CHECK(W > 0 && range_step(W, 304, 6) * 304 >= W && range_step(W, 304, 6) * 304 - W < 304);
  const int64_t c = tile_cost(big, s, big.tiles(16) - 1);
  CHECK(cut_block(c - 1, c, 2147483647 / 64 + 1, 6) <= 2147483647 / 64 + 1);
  puts("ok");
}
"""


def test_plan(tmp_path):
    src = tmp_path / "plan.cpp"
    src.write_text(PROG)
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o",
                    str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout.strip() == "ok"
