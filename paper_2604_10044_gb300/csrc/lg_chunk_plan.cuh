// How lg_chunk_attend's work is divided, in closed form, so that every CTA finds its share from the
// lengths alone.
//
// An item is (sequence, kv-head, tile): the g query heads of `tok` consecutive new tokens.  Its
// cost is the rows its queries can see plus kItemCost, a linear function of the tile (constant once
// a window fills), so the cost of a sequence's first t tiles is a closed form.  The items stand in
// one line, ordered by sequence, kv-head and tile, W cost units long, and each of G CTAs takes
// ceil(W / G) of it (or a block's rows, if that is more).  An item cut by such a bound is shared: its
// key blocks divide in proportion, each CTA's part is a piece, and a second kernel merges the pieces
// (of partial results in the workspace: slot 0 of a CTA for an item that began before its range,
// slot 1 for one that ends after it).
//
// Many items of a kv-head read the same rows.  One after the other on one CTA they read them from
// HBM once each, when the caches of all kv-heads together pass the L2; so the tiles of a kv-head can
// be dealt to `lanes` lines, tile t of kv-head h to line (t + h) mod lanes, each walked by G / lanes
// CTAs.  `lanes` divides G and the kv-heads, so a line holds every residue of a sequence's tiles
// equally often and all have the same length W; CTAs at the same place of each read the same
// kv-head's rows at about the same time.
#pragma once
#include <stdint.h>

#ifndef __CUDACC__
#define __host__
#define __device__
#define __forceinline__ inline
#endif

namespace lg {

// Cost of an item beside its rows: queries in, results out (in rows of keys).
constexpr int kItemCost = 96;

struct ChunkShape {
  int tok;     // tokens of a tile
  int bn2;     // log2 of the rows of a key block
  int window;  // 0: none
  int sink;
  int lanes2;  // log2 of the lines
};

// the sequences' numbers: rows n in the cache, m of them new
struct ChunkSeq {
  int n, m;
  __host__ __device__ __forceinline__ int tiles(int tok) const {
    return (unsigned)m / (unsigned)tok + ((unsigned)m % (unsigned)tok != 0);
  }
};

__host__ __device__ __forceinline__ int64_t plan_min(int64_t a, int64_t b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int64_t plan_max(int64_t a, int64_t b) { return a > b ? a : b; }

// a / b of numbers that mostly fit 32 bits (a 64-bit division takes some 100 instructions)
__host__ __device__ __forceinline__ int64_t plan_div(int64_t a, int64_t b) {
  if (((uint64_t)a | (uint64_t)b) >> 32 == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// rows tile t's queries see: first query row `first`, last `last`; rows [0, sinks) and [lo, last]
struct TileRows {
  int first, last, lo, sinks;
};

__host__ __device__ __forceinline__ TileRows tile_rows(const ChunkSeq &q, const ChunkShape &s,
                                                       int t) {
  TileRows r;
  r.first = q.n - q.m + t * s.tok;
  r.last = q.n - q.m + (int)plan_min(q.m, (int64_t)(t + 1) * s.tok) - 1;
  r.lo = s.window ? (int)plan_max(0, (int64_t)r.first + 1 - s.window) : 0;
  r.sinks = (int)plan_min(s.sink, r.lo);
  return r;
}

__host__ __device__ __forceinline__ int64_t tile_cost(const ChunkSeq &q, const ChunkShape &s,
                                                      int t) {
  const TileRows r = tile_rows(q, s, t);
  return (int64_t)r.last + 1 - r.lo + r.sinks + kItemCost;
}

// the first tile of a kv-head in line `lane`; the others follow `lanes` apart
__host__ __device__ __forceinline__ int first_tile(const ChunkShape &s, int lane, int kvh) {
  return (lane - kvh) & ((1 << s.lanes2) - 1);
}
__host__ __device__ __forceinline__ int lane_tiles(const ChunkSeq &q, const ChunkShape &s, int r) {
  const int tiles = q.tiles(s.tok);
  return tiles > r ? ((tiles - r - 1) >> s.lanes2) + 1 : 0;
}

// cost of the first k tiles of r, r + lanes, .., 0 <= k <= lane_tiles
__host__ __device__ __forceinline__ int64_t tiles_cost(const ChunkSeq &q, const ChunkShape &s, int r,
                                                       int k) {
  if (k <= 0) return 0;
  int64_t extra = 0;
  const int t = r + ((k - 1) << s.lanes2);
  if (t == q.tiles(s.tok) - 1) {  // the last tile may be short
    extra = tile_cost(q, s, t);
    if (--k == 0) return extra;
  }
  // full tiles t = r + j lanes, j < k: (n - m + (t + 1) tok) + kItemCost - max(0, a + t tok)
  const int64_t K = k, step = (int64_t)s.tok << s.lanes2, at = (int64_t)r * s.tok;
  int64_t sum = K * ((int64_t)q.n - q.m + kItemCost + at + s.tok) + step * (K * (K - 1) / 2);
  if (s.window) {
    const int64_t a = (int64_t)q.n - q.m + 1 - s.window - s.sink + at;
    const int64_t j0 = a >= 0 ? 0 : -a >= K * step ? K : plan_div(-a + step - 1, step);
    if (j0 < K) sum -= (K - j0) * a + step * ((K * (K - 1) - j0 * (j0 - 1)) / 2);
  }
  return sum + extra;
}

// cost of all tiles of a kv-head, which is that of `lanes` kv-heads in a line
__host__ __device__ __forceinline__ int64_t head_cost(const ChunkSeq &q, ChunkShape s) {
  s.lanes2 = 0;
  return tiles_cost(q, s, 0, q.tiles(s.tok));
}

// a tile's key blocks: block i of `count` holds the rows from block_row(i)
struct TileBlocks {
  int sink_blocks, skip, count;
  __host__ __device__ __forceinline__ int index(int i) const {
    return i < sink_blocks ? i : i + skip;
  }
};

__host__ __device__ __forceinline__ TileBlocks tile_blocks(const TileRows &r, int bn2) {
  TileBlocks b;
  const int w0 = r.lo >> bn2, w1 = (r.last >> bn2) + 1;
  b.sink_blocks = (int)(((int64_t)r.sinks + (1 << bn2) - 1) >> bn2);
  if (b.sink_blocks > w0) b.sink_blocks = w0;  // a block of both kinds counts once
  b.skip = w0 - b.sink_blocks;
  b.count = b.sink_blocks + w1 - w0;
  return b;
}

// The blocks, by their number among the tile's, that hide no row from any of its queries and hold
// none past the rows: the run [open0, open1) between the window's (hidden rows end at last - window)
// and the queries' own rows.  (A block with sinks may hide nothing either; it counts as hiding.)
__host__ __device__ __forceinline__ void open_blocks(const TileRows &r, const ChunkShape &s,
                                                     const TileBlocks &b, int &open0, int &open1) {
  const int64_t bn = (int64_t)1 << s.bn2;
  const int64_t from = s.window ? plan_max(0, (int64_t)r.last - s.window + 1) : 0;
  const int lo = (int)((from + bn - 1) >> s.bn2), hi = (int)(((int64_t)r.first + 1) >> s.bn2);
  open0 = lo - b.skip;
  open1 = hi > lo ? hi - b.skip : open0;
}

// cost units of a CTA of G: CTA c takes [c step, (c + 1) step) of the line, up to its end W; a block's
// rows at least, as a smaller share would leave CTAs without a block and the merge with empty parts
// (two blocks at least measured the same on short caches and slower on short prompts)
__host__ __device__ __forceinline__ int64_t range_step(int64_t W, int G, int bn2) {
  return plan_max(plan_div(W + G - 1, G), (int64_t)1 << bn2);
}

// blocks before a cut at cost unit y of an item: in whole blocks of the rows that the units stand
// for, the item's own cost first
__host__ __device__ __forceinline__ int cut_block(int64_t y, int64_t cost, int count, int bn2) {
  if (y >= cost) return count;
  const int64_t rows = y - kItemCost + ((1 << bn2) >> 1);
  return rows <= 0 ? 0 : (int)plan_min(rows >> bn2, count);
}

}  // namespace lg
