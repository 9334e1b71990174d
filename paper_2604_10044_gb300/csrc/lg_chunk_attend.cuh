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
  float *part;             // [2 G][d / 4][rows][4] partial sums, [2 G][rows][2] maxima and
                           // normalisers, then [G] ChunkCut
  int64_t S_total;
  int64_t cache_rows;      // L * H_kv * S_total
  int layer, batch, H_kv, g, T, max_new, max_len;
  int rows;                // of an item: tok * g rounded up to whole query tiles
  float qscale;            // softmax scale * log2(e)
  ChunkShape shape;
};

// a CTA's share: cost units [y0, y1) of its line of W, and the item that y0 falls into
struct ChunkShare {
  int64_t y0, y1, W, step;
  int64_t x;         // where the item starts in the line
  int64_t slot;      // its sequence's first cache slot
  ChunkSeq q;
  int b, off;        // off: its sequence's first token row
  int kvh, t;
  int lane;          // the line
};

// The share of CTA `cta` of G, which may be empty; false when it starts at the end of the line, the
// device status is set or a length is out of its bounds (recorded).  Every lane of a warp calls it;
// a batch of at most 32 is read once, in one round trip.  ONE: no sequence has more than one tile,
// and there is one line.
template <bool ONE>
__device__ __forceinline__ bool chunk_share(const ChunkAttendArgs &a, int cta, int G,
                                            ChunkShare &sh) {
  const int lane = threadIdx.x & 31, ctas = ONE ? G : G >> a.shape.lanes2;
  sh.lane = ONE ? 0 : cta / ctas;
  bool bad = false;
  int off = 0;
  int64_t slot = 0, c = 0, head = 0;
  ChunkSeq q{0, 0};
  auto load = [&](int b) {  // a lane's sequence, and its cost in the line: `head` a kv-head (or as many
    c = head = 0;           // as there are lines)
    if (b >= a.batch) return;
    off = a.off[b];
    const int end = a.off[b + 1];
    q = ChunkSeq{a.len[b], end - off};
    slot = a.seq_off[b];
    if (q.n < 0 || q.n > a.max_len || q.m < 0 || q.m > a.max_new || q.m > q.n || off < 0 ||
        end > a.T) {
      bad = true;
    } else {
      head = !ONE ? head_cost(q, a.shape) : q.m ? tile_cost(q, a.shape, 0) : 0;
      c = (ONE ? a.H_kv : a.H_kv >> a.shape.lanes2) * head;
    }
  };
  auto scan = [&](int64_t v) {  // inclusive prefix over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    return v;
  };
  auto range = [&] {
    const int k = ONE ? cta : cta - sh.lane * ctas;
    sh.step = range_step(sh.W, ctas, a.shape.bn2);
    sh.y0 = plan_min(sh.W, k * sh.step);
    sh.y1 = plan_min(sh.W, sh.y0 + sh.step);
    return sh.y0 < sh.W;
  };
  auto item = [&](int64_t per) {  // of sequence sh.b, which starts at sh.x
    const ChunkSeq q = sh.q;
    const int k = (int)plan_div(sh.y0 - sh.x, per);
    sh.x += k * per;
    sh.kvh = k;
    sh.t = 0;
    if (ONE) return;
    if (a.shape.lanes2) {  // which of the group's kv-heads: a lane each
      const int lanes = 1 << a.shape.lanes2;
      sh.kvh = k * lanes;
      const int r = first_tile(a.shape, sh.lane, sh.kvh + lane);
      const int64_t mine = lane < lanes ? tiles_cost(q, a.shape, r, lane_tiles(q, a.shape, r)) : 0;
      const int64_t incl = scan(mine);
      const int f = __ffs((int)__ballot_sync(0xffffffffu, sh.x + incl > sh.y0)) - 1;
      sh.x += __shfl_sync(0xffffffffu, incl - mine, f);
      sh.kvh += f;
    }
    // the last tile whose start is <= y0, among 32 at a time
    const int r = first_tile(a.shape, sh.lane, sh.kvh);
    const int64_t x0 = sh.x;
    int lo = 0;
    for (int n = lane_tiles(q, a.shape, r); n > 1;) {
      const int step = (n + 31) >> 5, i = lane * step;
      const int64_t start = x0 + (i < n ? tiles_cost(q, a.shape, r, lo + i) : 0);
      const int f = 31 - __clz((int)__ballot_sync(0xffffffffu, i < n && start <= sh.y0));
      sh.x = __shfl_sync(0xffffffffu, start, f);
      lo += f * step;
      n = (int)plan_min(step, n - f * step);
    }
    sh.t = r + (lo << a.shape.lanes2);
  };
  const bool stop = lane == 0 && status_bad(a.status);
  if (a.batch == 1) {  // nothing to search (the shortest call's latency is mostly this and its like)
    load(0);
    if (bad) set_status(a.status, LG_ERR_CAPACITY);
    if (__any_sync(0xffffffffu, bad || stop)) return false;
    sh.W = c;
    sh.x = 0;
    sh.slot = slot;
    sh.q = q;
    sh.off = off;
    sh.b = 0;
    if (!range()) return false;
    item(head);
    return true;
  }
  load(lane);
  int64_t incl = scan(c);
  sh.W = __shfl_sync(0xffffffffu, incl, 31);
  if (a.batch > 32) {
    int64_t mine = 0;
    for (int b = 32 + lane; b < a.batch; b += 32) {
      load(b);
      mine += c;
    }
    sh.W += __shfl_sync(0xffffffffu, scan(mine), 31);
    load(lane);
  }
  if (bad) set_status(a.status, LG_ERR_CAPACITY);
  if (__any_sync(0xffffffffu, bad || stop)) return false;
  if (!range()) return false;
  int64_t base = 0;
  for (int b0 = 0;; b0 += 32) {
    if (b0 > 0) {
      load(b0 + lane);
      incl = scan(c);
    }
    const unsigned past = __ballot_sync(0xffffffffu, base + incl > sh.y0);
    if (past) {
      const int f = __ffs((int)past) - 1;
      sh.x = base + __shfl_sync(0xffffffffu, incl - c, f);
      sh.slot = __shfl_sync(0xffffffffu, slot, f);
      sh.q.n = __shfl_sync(0xffffffffu, q.n, f);
      sh.q.m = __shfl_sync(0xffffffffu, q.m, f);
      sh.off = __shfl_sync(0xffffffffu, off, f);
      sh.b = b0 + f;
      item(__shfl_sync(0xffffffffu, head, f));
      return true;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
}

// The walk along a CTA's share, piece by piece.
template <bool ONE>
struct ChunkWalk {
  int b, kvh, t, tiles, lane;
  ChunkSeq q;
  int off;           // first token row of the sequence
  int64_t slot0;     // first cache slot of the sequence
  int64_t row0;      // first cache row of the (layer, kv-head, sequence)
  int64_t x, cost;   // the item's start in the line, and its cost
  int64_t y0, y1;
  TileRows rows;
  TileBlocks blocks;
  int blk0, blk1;    // the piece's key blocks

  __device__ __forceinline__ void load_item(const ChunkAttendArgs &a) {
    row0 = ((int64_t)a.layer * a.H_kv + kvh) * a.S_total + slot0;
    rows = tile_rows(q, a.shape, t);
    cost = tile_cost(q, a.shape, t);
    blocks = tile_blocks(rows, a.shape.bn2);
    blk0 = cut_block(y0 - x, cost, blocks.count, a.shape.bn2);
    blk1 = cut_block(y1 - x, cost, blocks.count, a.shape.bn2);
  }
  // the item that the share's start falls into
  __device__ __forceinline__ void start(const ChunkAttendArgs &a, const ChunkShare &sh) {
    b = sh.b;
    y0 = sh.y0;
    y1 = sh.y1;
    q = sh.q;
    off = sh.off;
    slot0 = sh.slot;
    lane = sh.lane;
    x = sh.x;
    kvh = sh.kvh;
    t = sh.t;
    tiles = ONE ? 1 : q.tiles(a.shape.tok);
    load_item(a);
  }
  __device__ __forceinline__ bool done() const { return x >= y1; }
  __device__ __forceinline__ void next(const ChunkAttendArgs &a) {
    x += cost;
    if (x >= y1) return;
    t += ONE ? 1 : 1 << a.shape.lanes2;
    while (t >= tiles) {  // (the line goes on, so there is another item)
      if (++kvh == a.H_kv) {
        kvh = 0;
        ++b;
        off = a.off[b];
        q = ChunkSeq{a.len[b], a.off[b + 1] - off};
        slot0 = a.seq_off[b];
        tiles = ONE ? q.m > 0 : q.tiles(a.shape.tok);
      }
      t = ONE ? 0 : first_tile(a.shape, lane, kvh);
    }
    load_item(a);
  }
  __device__ __forceinline__ bool whole() const { return blk0 == 0 && blk1 == blocks.count; }
  __device__ __forceinline__ int slot() const { return x < y0 ? 0 : 1; }
  __device__ __forceinline__ int tokens(const ChunkAttendArgs &a) const {
    return (int)plan_min(a.shape.tok, q.m - t * a.shape.tok);
  }
};

// four elements (4 e ..) of row r of a partial result: rows side by side, so that a warp whose lanes
// hold a row each writes and reads whole stretches
__device__ __forceinline__ float4 *part_at(const ChunkAttendArgs &a, int d, int cta, int slot, int e,
                                           int r) {
  return (float4 *)a.part + (((int64_t)cta * 2 + slot) * (d / 4) + e) * a.rows + r;
}

__device__ __forceinline__ float2 *part_ml(const ChunkAttendArgs &a, int d, int G, int cta,
                                           int slot, int r) {
  return (float2 *)(a.part + (int64_t)G * 2 * a.rows * d) + ((int64_t)cta * 2 + slot) * a.rows + r;
}

// What the merge has to know of the item that a CTA's start cuts, written by that CTA.
struct ChunkCut {
  int64_t in, step, cost;  // cost units: of the start in the item, of a CTA, of the item
  int parts;               // CTAs from the one before on that have a part; 0: nothing to merge
  int blocks, used, tok0;  // key blocks and query rows of the item, its first token row
  int kvh, pad;
};

__device__ __forceinline__ ChunkCut *cut_at(const ChunkAttendArgs &a, int d, int G, int cta) {
  return (ChunkCut *)(a.part + (int64_t)G * 2 * a.rows * (d + 2)) + cta;
}

// One thread of every CTA calls it: `work` as chunk_share gave it, w at its start.
template <bool ONE>
__device__ __forceinline__ void put_cut(const ChunkAttendArgs &a, int d, int G, int cta, bool work,
                                        const ChunkShare &sh, const ChunkWalk<ONE> &w) {
  ChunkCut c = {};
  // the start falls inside the item, and no earlier one does
  if (work && w.x < sh.y0 && sh.y0 - sh.step <= w.x) {
    c.in = sh.y0 - w.x;
    c.step = sh.step;
    c.cost = w.cost;
    c.parts = 2;
    for (int64_t y = c.in + c.step; y < c.cost; y += c.step) ++c.parts;
    c.blocks = w.blocks.count;
    c.used = w.tokens(a) * a.g;
    c.tok0 = w.off + w.t * a.shape.tok;
    c.kvh = w.kvh;
  }
  *cut_at(a, d, G, cta) = c;
}

__device__ __forceinline__ bool row_sees(const TileRows &r, const ChunkShape &s, int query_row,
                                         int i) {
  return i <= query_row && (s.window == 0 || i > query_row - s.window || i < s.sink);
}

// bf16: the kernel on the tensor cores (lg_chunk_attend_tc.cu)
ChunkGrid chunk_grid_tc(int d, int g, int max_new);
cudaError_t launch_chunk_attend_tc(const ChunkAttendArgs &a, int d, int G, cudaStream_t s);

cudaError_t launch_chunk_attend_few(const ChunkAttendArgs &a, int d, int G, cudaStream_t s);

// the merge of items that several CTAs share (lg_chunk_attend.cu)
cudaError_t launch_chunk_merge(const ChunkAttendArgs &a, int dtype, int d, int G, cudaStream_t s);

}  // namespace lg
