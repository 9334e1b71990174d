// What the kernels of lg_chunk_attend share: arguments, a CTA's share of the line of items
// (lg_chunk_plan.cuh), the walk along it, and the partial results in the workspace.
#pragma once
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lg_chunk_plan.cuh"
#include "lg_common.cuh"
#include "lg_internal.h"

namespace lg {

struct ChunkAttendArgs {
  const void *K, *V;       // cache [L][H_kv][S_total][d]
  const void *q;           // [T][H_q][d]
  void *out;               // [T][H_q][d]
  const int64_t *seq_off;  // [batch]
  const int32_t *len;      // [batch]
  const int32_t *off;      // [batch + 1]
  int32_t *status;
  float *part;             // [2 G][rows][d] partial sums, then [2 G][rows][2] maxima and normalisers
  int64_t S_total;
  int64_t cache_rows;      // L * H_kv * S_total
  int layer, batch, H_kv, g, T, max_new, max_len;
  int rows;                // of an item: tok * g rounded up to whole query tiles
  float qscale;            // softmax scale * log2(e)
  ChunkShape shape;
};

// a CTA's share: cost units [y0, y1) of the line, and the sequence that y0 falls into
struct ChunkShare {
  int64_t y0, y1, W, x;  // W: the whole line; x: where sequence b starts in it
  int b;
};

__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkAttendArgs &a, int b, int &off) {
  off = a.off[b];
  return ChunkSeq{a.len[b], a.off[b + 1] - off};
}

__device__ __forceinline__ int64_t seq_cost(const ChunkAttendArgs &a, const ChunkSeq &q) {
  return a.H_kv * tiles_cost(q, a.shape, q.tiles(a.shape.tok));
}

// The share of CTA `cta` of G, which may be empty; false (for every thread) when it starts at the
// end of the line, the device status is set or a length is out of its bounds (recorded).  Every
// thread of the CTA calls it; the lengths are read once for a batch of at most NT.
template <int NT>
__device__ bool chunk_share(const ChunkAttendArgs &a, int cta, int G, ChunkShare &sh) {
  __shared__ int64_t s_warp[NT / 32];
  __shared__ ChunkShare s_share;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  bool bad = false, stop = tid == 0 && status_bad(a.status);
  int64_t mine = 0, first = 0;  // this thread's sequences; the one of the first round
  for (int b = tid; b < a.batch; b += NT) {
    int off;
    const ChunkSeq q = chunk_seq(a, b, off);
    if (q.n < 0 || q.n > a.max_len || q.m < 0 || q.m > a.max_new || q.m > q.n || off < 0 ||
        (int64_t)off + q.m > a.T) {
      bad = true;
      continue;
    }
    const int64_t cost = seq_cost(a, q);
    if (b == tid) first = cost;
    mine += cost;
  }
  if (bad) set_status(a.status, LG_ERR_CAPACITY);
  if (__syncthreads_or(bad || stop)) return false;

  auto scan = [&](int64_t v, int64_t &total) {  // inclusive prefix over the CTA's threads
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < NT / 32; ++w) {
      if (w < warp) before += s_warp[w];
      total += s_warp[w];
    }
    return v + before;
  };
  int64_t W, incl = scan(mine, W);
  const int64_t y0 = range_bound(W, cta, G), y1 = range_bound(W, cta + 1, G);
  if (y0 >= W) return false;
  int64_t base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += NT) {
    int64_t cost = first, total = W;
    if (a.batch > NT) {  // rounds of NT sequences in order
      int off;
      cost = 0;
      if (b0 + tid < a.batch) cost = seq_cost(a, chunk_seq(a, b0 + tid, off));
      incl = scan(cost, total);
    }
    const int64_t x = base + incl - cost;
    if (y0 >= x && y0 < x + cost) s_share = ChunkShare{y0, y1, W, x, b0 + tid};
    base += total;
    if (y0 < base) break;
  }
  __syncthreads();
  sh = s_share;
  return true;
}

// The walk along a CTA's share, piece by piece; every role of a CTA walks by itself.
struct ChunkWalk {
  int b, kvh, t, tiles;
  ChunkSeq q;
  int off;           // first token row of the sequence
  int64_t row0;      // first cache row of the (layer, kv-head, sequence)
  int64_t x, cost;   // the item's start in the line, and its cost
  int64_t per_head;  // cost of a kv-head's tiles
  int64_t y0, y1;
  TileRows rows;
  TileBlocks blocks;
  int blk0, blk1;    // the piece's key blocks

  __device__ __forceinline__ void load_seq(const ChunkAttendArgs &a) {
    q = chunk_seq(a, b, off);
    tiles = q.tiles(a.shape.tok);
  }
  __device__ __forceinline__ void load_item(const ChunkAttendArgs &a) {
    row0 = ((int64_t)a.layer * a.H_kv + kvh) * a.S_total + a.seq_off[b];
    rows = tile_rows(q, a.shape, t);
    cost = tile_cost(q, a.shape, t);
    blocks = tile_blocks(rows, a.shape.bn2);
    blk0 = cut_block(y0 - x, cost, blocks.count, a.shape.bn2);
    blk1 = cut_block(y1 - x, cost, blocks.count, a.shape.bn2);
  }
  // the item that cost unit y falls into, y in sequence sh.b
  __device__ __forceinline__ void start(const ChunkAttendArgs &a, const ChunkShare &sh, int64_t y) {
    b = sh.b;
    y0 = sh.y0;
    y1 = sh.y1;
    load_seq(a);
    per_head = tiles_cost(q, a.shape, tiles);
    kvh = (int)plan_div(y - sh.x, per_head);
    const int64_t in = y - sh.x - kvh * per_head;
    t = tile_at(q, a.shape, in);
    x = sh.x + kvh * per_head + tiles_cost(q, a.shape, t);
    load_item(a);
  }
  __device__ __forceinline__ bool done() const { return x >= y1; }
  __device__ __forceinline__ void next(const ChunkAttendArgs &a) {
    x += cost;
    if (x >= y1) return;
    if (++t == tiles) {
      t = 0;
      if (++kvh == a.H_kv) {
        kvh = 0;
        do {
          ++b;
          load_seq(a);
        } while (tiles == 0);
      }
    }
    load_item(a);
  }
  __device__ __forceinline__ bool whole() const { return blk0 == 0 && blk1 == blocks.count; }
  __device__ __forceinline__ int slot() const { return x < y0 ? 0 : 1; }
  __device__ __forceinline__ int tokens(const ChunkAttendArgs &a) const {
    return (int)plan_min(a.shape.tok, q.m - t * a.shape.tok);
  }
};

__device__ __forceinline__ float *part_row(const ChunkAttendArgs &a, int d, int cta, int slot,
                                           int r) {
  return a.part + (((int64_t)cta * 2 + slot) * a.rows + r) * d;
}

__device__ __forceinline__ float2 *part_ml(const ChunkAttendArgs &a, int d, int G, int cta,
                                           int slot, int r) {
  return (float2 *)(a.part + (int64_t)G * 2 * a.rows * d) + ((int64_t)cta * 2 + slot) * a.rows + r;
}

__device__ __forceinline__ bool row_sees(const TileRows &r, const ChunkShape &s, int query_row,
                                         int i) {
  return i <= query_row && (s.window == 0 || i > query_row - s.window || i < s.sink);
}

// bf16: the kernel on the tensor cores (lg_chunk_attend_tc.cu)
ChunkGrid chunk_grid_tc(int g, int max_new);
cudaError_t launch_chunk_attend_tc(const ChunkAttendArgs &a, int d, int G, cudaStream_t s);

cudaError_t launch_chunk_attend_few(const ChunkAttendArgs &a, int d, int G, cudaStream_t s);

// the merge of items that several CTAs share (lg_chunk_attend.cu)
cudaError_t launch_chunk_merge(const ChunkAttendArgs &a, int dtype, int d, int G, cudaStream_t s);

}  // namespace lg
