// How the work of attention over a 4-bit cache is divided, in closed form, so that every CTA finds
// its share from the lengths alone.
//
// An item is (sequence, kv-head, tile of query rows).  The items of a layer stand in one line,
// ordered like that; an item takes the key blocks that any query of its sequence sees, and
// kQ4ItemUnits more for its start and end, so all items of a sequence take the same.  Each of G
// CTAs takes ceil(W / G) units of the line's W.  Its share of an item's blocks is a piece; an item
// of which one piece has every block is finished by that CTA, the pieces of the others go through
// the workspace (slot 0 of a CTA for an item that began before its share, slot 1 for one that
// begins in it) to a second kernel.
#pragma once
#include "lg_chunk_plan.cuh"

namespace lg {

constexpr int kQ4Bn2 = 7;        // log2 of the rows of a key block
constexpr int kQ4ItemUnits = 2;  // of an item beside its blocks

struct Q4Shape {
  int rows, g;       // query rows of an item, query heads of a kv-head
  int window, sink;
  int H_kv;
};

__host__ __device__ __forceinline__ int q4_tiles(const ChunkSeq &q, const Q4Shape &s) {
  return q.m ? (int)(((int64_t)q.m * s.g + s.rows - 1) / s.rows) : 0;
}

// the rows that the queries of tile t see, and how many query rows it has
__host__ __device__ __forceinline__ TileRows q4_rows(const ChunkSeq &q, const Q4Shape &s, int t,
                                                     int &used) {
  const int64_t first = (int64_t)t * s.rows;
  used = (int)plan_min(s.rows, (int64_t)q.m * s.g - first);
  TileRows r;
  r.first = q.n - q.m + (int)(first / s.g);
  r.last = q.n - q.m + (int)((first + used - 1) / s.g);
  r.lo = s.window ? (int)plan_max(0, (int64_t)r.first + 1 - s.window) : 0;
  r.sinks = (int)plan_min(s.sink, r.lo);
  return r;
}

// units of an item: blocks of a tile that had all queries, and no tile has more
__host__ __device__ __forceinline__ int q4_units(const ChunkSeq &q, const Q4Shape &s) {
  if (q.m == 0) return 0;
  TileRows r;
  r.first = q.n - q.m;
  r.last = q.n - 1;
  r.lo = s.window ? (int)plan_max(0, (int64_t)r.first + 1 - s.window) : 0;
  r.sinks = s.window ? s.sink : 0;  // (a later tile's window may leave more sinks before it)
  const int w0 = r.lo >> kQ4Bn2, w1 = (r.last >> kQ4Bn2) + 1;
  const int64_t sinks = ((int64_t)r.sinks + (1 << kQ4Bn2) - 1) >> kQ4Bn2;
  return (int)plan_min(sinks + w1 - w0, w1) + kQ4ItemUnits;
}

__host__ __device__ __forceinline__ int64_t q4_seq_units(const ChunkSeq &q, const Q4Shape &s) {
  return (int64_t)s.H_kv * q4_tiles(q, s) * q4_units(q, s);
}

// blocks before unit u of an item that has `count`
__host__ __device__ __forceinline__ int q4_cut(int64_t u, int count) {
  return (int)plan_max(0, plan_min(u - kQ4ItemUnits, count));
}

}  // namespace lg
