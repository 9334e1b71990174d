// Attention of few query rows of a kv-head (a token, or some drafted tokens, a sequence) over a
// 4-bit cache, with the statistics that the guard reads of a single token.
//
// A warp takes 16 rows of keys and values at a time through mma.sync (M = 16 keys or 16 elements, N
// = 8 query rows, K = 16), and a value is never formed from its code and parameters:
//   scores   q . k = sum over groups of (s_g sum_e q_e c_e) + sum_g lo_g sum_{e in g} q_e.  A code
//            masked out of its word is a bf16 number as it stands: the low eight bits of one count
//            in units of 2^-133 (its subnormal numbers, and the first normal ones), so bits 0-3 are
//            c and bits 4-7 16 c of them.  The queries bring the factor, 2^120 over the power of
//            two of the row's largest element (and a sixteenth of that for the 16 c); both are
//            exact, so are the products.  The groups' sums are joined by the rows' scales in fp32;
//            the least values are one more product, with sums of q in three bf16 terms (two left
//            the statistics 2^-17 of |lo| |sum q| off, 1e-6 of a score, for the same time).
//   results  sum_k p_k v_k = sum_k (p_k s_kg)(c - 8) + sum_k p_k lo_kg + 8 sum_k p_k s_kg: the
//            second operand is the weights times a group's scales, rounded to bf16; the last two
//            are one product whose first operand is the rows' parameters.  One fused operation
//            turns the masked code into (c - 8) / 64 or / 4: with codes about zero sums stay small
//            beside what the matrix unit drops of them, and a weight's second rounding meets |c -
//            8|, not c.  The two roundings leave 2.8e-3 of random values' results, of which the
//            result's own is 1.7e-3; weights and products in two terms leave nothing beside that,
//            for 17 % of the time (64 sequences 93 and 108 us, 262143 rows 66 and 77): not taken, as
//            the codes are off by some 8 % of the spread of a group's values.
// Codes and parameters come by ldmatrix: a 16-byte piece of a row is a group (two of them, for d =
// 64), and transposed a register holds a half word of codes of two neighbouring keys, which is a
// pair of each of its nibbles.  For d = 64 a product of the scores takes one group of the two, the
// other's queries being zero, and of the results half of the rows are of use.
//
// Weights are 2^(z - m) with a maximum m that may lag: it is formed anew only when a score passes
// it by 8, so a tile asks one vote.  Every warp has its own m and sums; the CTA's four are merged
// at its end, and the CTAs of an item by a second kernel (or, as a cluster, by themselves:
// q4_grid).
//
// Every warp copies its own 32 rows a block (bulk copies into a ring of its own), so warps never
// wait for one another.
//
// GB300, 8 kv-heads of 128, 4 query heads each: 64 sequences of 1024 to 16381 rows (477 MB) 84 us
// in this kernel, 5.7 TB/s, and 92 with the merge; one of 262143 rows (336 MB) 58 and 66; what
// bounds it is issue: the warps issue in 55 to 60 % of the cycles, half of that masks and fused
// conversions of codes, while HBM is at 83 %.  Steps that led here: codes as 128 + c with the 128
// taken off afterwards 166 us (64 sequences); codes as they stand and ldmatrix 144; 32 rows a warp
// and stage 110; equal shares of a line 95; three CTAs an SM of 168 registers instead of four of
// 128 (whose spills cost more than their warps gave) 91.  Not kept: five CTAs an SM 129; one
// product of 16 rows at a time through the softmax 98; three and four stages the same and 135.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lg_q4.cuh"

namespace lg {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kSub = 32;             // rows of a warp's tile, 16 a product
constexpr int kBn2 = kQ4Bn2;         // a CTA's block: kWarps tiles
constexpr int kClusterMost = 8;      // CTAs of a cluster
constexpr float kLazy = 8.f;         // log2 units that a weight may pass 1 by
constexpr float kHidden = -1e38f;    // score of a row that a query does not see
constexpr float kNone = -1e30f;      // maximum of a query that has seen nothing
static_assert(kWarps * kSub == 1 << kBn2, "a tile a warp");

template <int D, int NT>
struct Q4Cfg {
  static constexpr int kRow = q4_row_bytes(D);
  static constexpr int kTile = kSub * kRow;         // of keys, or of values
  static constexpr int kCtas = NT == 1 ? 3 : 2;  // of an SM
  static constexpr int kStages = D == 64 ? 4 : NT == 1 ? 2 : NT == 2 ? 3 : 4;
  static constexpr int kJoint = NT <= 2 ? 2 : 1;  // products of 16 rows with one softmax step
  static constexpr int kRing = kWarps * kStages * 2 * kTile;
  static constexpr int kRows = 8 * NT;
  static constexpr int kOut = kWarps * kRows * (D + 1) * 4;  // the warps' results, for their merge
  static constexpr int kQ = NT > 2 ? NT * 4 * 32 * 16 : 0;   // fragments of q, unless in registers
  static constexpr int kPart = kRows * (D + 4) * 4;          // a CTA's results, for its cluster
  static constexpr int kSmem = (kRing > kOut + kPart ? kRing : kOut + kPart) + kQ;
};

// The 16-byte piece of a row that holds group gr, and whether word (or half word) i of it, of four
// (eight), belongs to the group.
template <int D>
__device__ __forceinline__ constexpr int piece_of(int gr) {
  return D == 128 ? gr : gr >> 1;
}
template <int D, int N>
__device__ __forceinline__ bool of_group(int gr, int i) {
  return D == 128 || i / (N / 2) == (gr & 1);
}

// the element of row r (g or g + 8) of result tile u of group gr: nibble 2u or 2u + 1 of half word
// g
template <int D>
__device__ __forceinline__ int value_element(int gr, int u, int g, int up) {
  return 8 * (4 * piece_of<D>(gr) + (g >> 1)) + 2 * (2 * u + up) + (g & 1);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t *)&h;
}

__device__ __forceinline__ uint32_t max_abs(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r =
      __hmax2(__habs2(*(const __nv_bfloat162 *)&a), __habs2(*(const __nv_bfloat162 *)&b));
  return *(const uint32_t *)&r;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
  return *(const uint32_t *)&r;
}

// masked codes, c or 16 c in units of 2^-133, to (c - 8) / 64 or (c - 8) / 4
__device__ __forceinline__ uint32_t centred(uint32_t raw, bool high) {
  const uint32_t by = 0x7f007f00u, less = high ? 0xc000c000u : 0xbe00be00u;  // 2^127; -2 or -1/8
  const __nv_bfloat162 r = __hfma2(*(const __nv_bfloat162 *)&raw, *(const __nv_bfloat162 *)&by,
                                   *(const __nv_bfloat162 *)&less);
  return *(const uint32_t *)&r;
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldmatrix2(uint32_t &a, uint32_t &b, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];"
               : "=r"(a), "=r"(b) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix2_trans(uint32_t &a, uint32_t &b, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];"
               : "=r"(a), "=r"(b) : "r"(at) : "memory");
}

// a half that is not finite, or whose key is past the last row, becomes zero
__device__ __forceinline__ uint32_t finite_pair(uint32_t x, bool keep0, bool keep1) {
  uint32_t mask = 0;
  if (keep0 && (x & 0x7f80u) != 0x7f80u) mask |= 0xffffu;
  if (keep1 && (x & 0x7f800000u) != 0x7f800000u) mask |= 0xffff0000u;
  return x & mask;
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// a partial result: [rows][D + 4], the sums and {m, l, sum p (z - m), suffix}; m the true maximum
template <int D>
__device__ __forceinline__ float *part_row(const Q4AttendArgs &a, int layer, int cta, int slot,
                                           int r) {
  return a.part + (((int64_t)layer * a.ctas + cta) * 2 + slot) * a.shape.rows * (int64_t)(D + 4) +
         r * (D + 4);
}

// A sequence's numbers; false where they are out of bounds.  Without offsets every sequence that
// has rows has one query, for its last.
__device__ __forceinline__ bool q4_seq(const Q4AttendArgs &a, int b, ChunkSeq &q, int &off) {
  q.n = a.len[b];
  off = a.off ? a.off[b] : b;
  q.m = a.off ? a.off[b + 1] - off : (q.n > 0 ? 1 : 0);
  return q.n >= 0 && q.n <= a.max_len && q.m >= 0 && q.m <= a.max_new && q.m <= q.n && off >= 0 &&
         off + q.m <= a.T;
}

__device__ __forceinline__ int64_t warp_scan(int64_t v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// The line's units W, and the sequence that CTA `cta`'s first unit falls into, with its start and
// its numbers (nothing where the CTA's share starts at the end of the line).  False when a number
// is out of bounds (recorded).  Every lane of a warp calls it; a batch of at most 32 is read once.
struct Q4Line {
  int64_t W, step;
  int64_t x;
  ChunkSeq q;
  int b, off;
};
__device__ __forceinline__ bool q4_line(const Q4AttendArgs &a, int cta, Q4Line &f) {
  const int lane = threadIdx.x & 31;
  ChunkSeq q{0, 0};
  int off = 0;
  bool bad = false;
  auto units = [&](int i) -> int64_t {
    if (i >= a.batch) return 0;
    if (!q4_seq(a, i, q, off)) {
      bad = true;
      return 0;
    }
    return q4_seq_units(q, a.shape);
  };
  f.x = 0;
  f.b = 0;
  const int64_t c0 = units(a.batch == 1 ? 0 : lane);
  int64_t s0 = c0;
  if (a.batch == 1) {  // nothing to search: the shortest call's latency is mostly this and its like
    f.W = c0;
  } else {
    s0 = warp_scan(c0, lane);
    f.W = __shfl_sync(0xffffffffu, s0, 31);
    if (a.batch > 32) {
      const ChunkSeq q0 = q;
      const int off0 = off;
      int64_t mine = 0;
      for (int i = 32 + lane; i < a.batch; i += 32) mine += units(i);
      f.W += __shfl_sync(0xffffffffu, warp_scan(mine, lane), 31);
      q = q0;
      off = off0;
    }
  }
  if (__any_sync(0xffffffffu, bad)) {
    if (threadIdx.x == 0) set_status(a.status, LG_ERR_CAPACITY);
    return false;
  }
  f.step = plan_max(1, plan_div(f.W + a.ctas - 1, a.ctas));
  f.q = q;
  f.off = off;
  const int64_t y0 = cta * f.step;
  if (a.batch == 1 || y0 >= f.W) return true;
  for (int i0 = 0;; i0 += 32) {
    const int64_t c = i0 ? units(i0 + lane) : c0;
    const int64_t incl = i0 ? warp_scan(c, lane) : s0;
    const unsigned past = __ballot_sync(0xffffffffu, f.x + incl > y0);
    if (past) {
      const int k = __ffs((int)past) - 1;
      f.x += __shfl_sync(0xffffffffu, incl - c, k);
      f.b = i0 + k;
      f.q.n = __shfl_sync(0xffffffffu, q.n, k);
      f.q.m = __shfl_sync(0xffffffffu, q.m, k);
      f.off = __shfl_sync(0xffffffffu, off, k);
      return true;
    }
    f.x += __shfl_sync(0xffffffffu, incl, 31);
  }
}

// What the merge has to know of the item that a CTA's start cuts, written by that CTA if no earlier
// start cuts the item.
struct Q4Cut {
  int64_t x0;    // the item's start in the line
  int64_t step;  // 0: nothing to merge
  int64_t head;  // its first query head's row in the outputs
  int units, count, used, row_1;
};
__device__ __forceinline__ Q4Cut *cut_at(const Q4AttendArgs &a, int d, int layer, int cta) {
  return (Q4Cut *)(a.part + (int64_t)a.n_layers * a.ctas * 2 * a.shape.rows * (d + 4)) +
         (int64_t)layer * a.ctas + cta;
}

template <int D, int NT, bool STATS, bool CL>
__global__ void __launch_bounds__(kThreads, (Q4Cfg<D, NT>::kCtas))
    q4_attend_kernel(Q4AttendArgs a) {
  using C = Q4Cfg<D, NT>;
  constexpr int kPieces = D / 32;  // 16-byte pieces of a row's codes
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t s_full[kWarps][C::kStages];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (lane == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(&s_full[warp][i], 1);
    mbar_fence_init();
  }
  __syncwarp();
  pdl_enter();
  // (CTAs of a cluster, which meet at barriers, may find another status each: they go on without
  // work)
  const bool bad = cta_status_bad(a.status);
  if (!CL && bad) return;
  const int layer = blockIdx.y, cta = blockIdx.x;  // (layer of the call)
  const int H_q = a.H_kv * a.g;
  float *s_o = (float *)smem;  // [warp][row][D + 1], the warps' results
  __shared__ float4 s_st[kWarps][8 * NT];
  struct {
    ChunkSeq q;
    TileRows rows;
    TileBlocks blocks;
    int kvh, tile, off, used;
  } w;
  int seq, units, tiles;
  int64_t x, y0, y1;  // the item's start in the line, the CTA's share
  if constexpr (CL) {  // a cluster an item
    unsigned item = blockIdx.x / (unsigned)a.cluster;
    tiles = (int)(((int64_t)a.max_new * a.g + a.shape.rows - 1) / a.shape.rows);
    w.tile = (int)(item % (unsigned)tiles);
    item /= (unsigned)tiles;
    w.kvh = (int)(item % (unsigned)a.H_kv);
    seq = (int)(item / (unsigned)a.H_kv);
    if (!q4_seq(a, seq, w.q, w.off)) {  // (the same in the cluster, as what returns below)
      if (tid == 0) set_status(a.status, LG_ERR_CAPACITY);
      return;
    }
    if (STATS && w.q.n == 0 && !bad && blockIdx.x % (unsigned)a.cluster == 0) {
      const int64_t head = ((int64_t)layer * a.T + w.off) * H_q + w.kvh * a.g;  // attends to nothing
      for (int e = tid; e < a.g * D / 2; e += kThreads) ((uint32_t *)a.out)[head * D / 2 + e] = 0u;
      if (tid < a.g) ((float4 *)a.stats)[head + tid] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
    if (w.tile >= q4_tiles(w.q, a.shape)) return;
    x = y0 = 0;
    y1 = units = 1;
  } else {
    Q4Line line;
    if (!q4_line(a, cta, line)) return;
    y0 = cta * line.step, y1 = plan_min(y0 + line.step, line.W);
    if (y0 >= y1) {
      if (tid == 0) cut_at(a, D, layer, cta)->step = 0;
      return;
    }
    seq = line.b;
    x = line.x;
    w.q = line.q;
    w.off = line.off;
    units = q4_units(w.q, a.shape), tiles = q4_tiles(w.q, a.shape);
    const int64_t k = plan_div(y0 - x, units);
    x += k * units;
    w.kvh = (int)plan_div(k, tiles);
    w.tile = (int)(k - (int64_t)w.kvh * tiles);
    if (tid == 0) {
      Q4Cut c = {};
      if (x < y0 && y0 - line.step <= x) {
        const TileRows rows = q4_rows(w.q, a.shape, w.tile, c.used);
        c.x0 = x;
        c.step = line.step;
        c.head = ((int64_t)layer * a.T + w.off) * H_q + w.kvh * a.g;
        c.units = units;
        c.count = tile_blocks(rows, kBn2).count;
        c.row_1 = w.tile * a.shape.rows;
      }
      *cut_at(a, D, layer, cta) = c;
    }
  }
  // this lane's row and 16-byte piece of an ldmatrix of four, and its row of one of two
  const uint32_t at4 = (lane & 15) * C::kRow + 16 * (lane >> 4);
  const uint32_t at2 = (lane & 15) * C::kRow + D / 2;
  uint8_t *ring = smem + warp * C::kStages * 2 * C::kTile;
  int st = 0, phase = 0;  // of the next block to be read: they go on over the pieces
  bool gave_up = false;

  for (; x < y1 && !gave_up; x += units) {
    w.rows = q4_rows(w.q, a.shape, w.tile, w.used);
    w.blocks = tile_blocks(w.rows, kBn2);
    int blk0, blk1;
    if constexpr (CL) {
      const int rank = (int)(blockIdx.x % (unsigned)a.cluster);
      blk0 = (int)((int64_t)rank * w.blocks.count / a.cluster);
      blk1 = bad ? blk0 : (int)((int64_t)(rank + 1) * w.blocks.count / a.cluster);
    } else {
      blk0 = q4_cut(y0 - x, w.blocks.count), blk1 = q4_cut(y1 - x, w.blocks.count);
    }
    if (CL || blk0 < blk1) {
      // this warp's copies: its rows of each block
      const int64_t row0 = ((int64_t)(a.layer0 + layer) * a.H_kv + w.kvh) * a.S_total + a.seq_off[seq];
      const uint8_t *gk = a.K + row0 * C::kRow, *gv = a.V + row0 * C::kRow;
      auto tile_row = [&](int i) { return (w.blocks.index(i) << kBn2) + warp * kSub; };
      auto copy = [&](int i, uint8_t *to, uint64_t *bar) {  // lane 0: block i into a stage
        const int r = tile_row(i);
        const int n = min(kSub, w.rows.last + 1 - r);
        if (n <= 0) return;
        const int bytes = n * C::kRow;
        const int64_t from = (int64_t)r * C::kRow;
        mbar_arrive_expect_tx(bar, 2 * bytes);
        bulk_load(to, gk + from, bytes, bar);
        bulk_load(to + C::kTile, gv + from, bytes, bar);
      };
      if (lane == 0)
        for (int k = 0, to = st; k < C::kStages && blk0 + k < blk1; ++k) {
          copy(blk0 + k, ring + to * 2 * C::kTile, &s_full[warp][to]);
          if (++to == C::kStages) to = 0;
        }

      // q as second operands, and its groups' sums in three terms for the least values
      const __nv_bfloat16 *q = (const __nv_bfloat16 *)a.q +
                               ((int64_t)layer * a.T + w.off) * H_q * D + (int64_t)w.kvh * a.g * D;
      const int row_1 = w.tile * a.shape.rows;  // the tile's first query row
      auto q_row = [&](int r) {  // row r of the item, or null
        r += row_1;
        return r < row_1 + w.used ? q + ((int64_t)(r / a.g) * H_q + r % a.g) * D : nullptr;
      };
      uint32_t qf[NT <= 2 ? NT : 1][4][4];
      uint4 *s_q = (uint4 *)(smem + C::kSmem - C::kQ);
      uint32_t sum_12[NT], sum_3[NT];
      float cm[NT][2];  // column 2t, 2t+1: what turns its sums into log2 units
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const __nv_bfloat16 *src = q_row(8 * nt + g);
        uint4 v[kPieces];  // words t of the pieces: eight elements each
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          v[j] = src ? *(const uint4 *)(src + 8 * (4 * j + t)) : make_uint4(0, 0, 0, 0);
          most = max_abs(max_abs(max_abs(most, v[j].x), max_abs(v[j].y, v[j].z)), v[j].w);
        }
        float big = fmaxf(bf16_low(most), bf16_high(most));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        // the power of two of the largest, kept where 2^120 over it is a number
        const int ex = min(max((int)(__float_as_uint(big) >> 23) - 127, -7), 114);
        const float up = __uint_as_float((uint32_t)(120 - ex + 127) << 23);
        // (a query whose products would leave fp32 or bf16 gives NaN)
        float mult = a.qscale * __uint_as_float((uint32_t)(13 + ex + 127) << 23);
        if (!(big < 0x1p121f) || mult == INFINITY) mult = __int_as_float(0x7fffffff);
        cm[nt][0] = __shfl_sync(0xffffffffu, mult, 8 * t);
        cm[nt][1] = __shfl_sync(0xffffffffu, mult, 8 * t + 4);
        const uint32_t up_even = pack_bf16(up, up), up_odd = pack_bf16(up * 0.0625f, up * 0.0625f);
        float mine = 0.f;
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
          const uint4 w4 = v[piece_of<D>(gr)];
          const uint32_t x[4] = {w4.x, w4.y, w4.z, w4.w};
          const bool in = of_group<D, 4>(gr, t);
          uint32_t f[4];
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // pair i of a word; odd ones meet 16 c
            f[i] = in ? mul_bf16x2(x[i], i & 1 ? up_odd : up_even) : 0u;
            sum += bf16_low(x[i]) + bf16_high(x[i]);
          }
          sum = in ? sum : 0.f;
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          if (t == gr) mine = sum * (up * 0x1p-120f) * 0x1p-13f;
          if constexpr (NT <= 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[nt][gr][i] = f[i];
          } else if (warp == 0) {
            s_q[(nt * 4 + gr) * 32 + lane] = make_uint4(f[0], f[1], f[2], f[3]);
          }
        }
        const float hi = __bfloat162float(__float2bfloat16_rn(mine));
        const float mid = __bfloat162float(__float2bfloat16_rn(mine - hi));
        sum_12[nt] = pack_bf16(hi, mid);
        sum_3[nt] = pack_bf16(mine - hi - mid, 0.f);
      }
      if constexpr (NT > 2) __syncthreads();

      const int low_max =
          a.shape.window ? (int)plan_max(0, (int64_t)w.rows.last + 1 - a.shape.window) : 0;
      const int suffix0 = w.q.n - a.suffix_w;  // (n and suffix_w are positive)
      auto last_seen = [&](int r) {            // the own row of the query of row r of the item
        return w.q.n - w.q.m + (min(r, w.used - 1) + row_1) / a.g;
      };
      auto low_seen = [&](int last) {
        return a.shape.window ? (int)plan_max(0, (int64_t)last + 1 - a.shape.window) : 0;
      };
      auto hides = [&](int r, int last, int low) {
        return r > last || (r < low && r >= a.shape.sink);
      };

      float o[NT][4][2][4] = {};
      // rows 2 gr: the weights times group gr's scales; rows 2 gr + 1: times its least values
      float ox[NT][4] = {};
      float m[NT][2], top[NT][2], l[NT][2], hs[NT][2], sf[NT][2];  // top: the largest score, less m
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          m[nt][c] = top[nt][c] = kNone;
          l[nt][c] = hs[nt][c] = sf[nt][c] = 0.f;
        }

      constexpr int J = C::kJoint;
      for (int i = blk0; i < blk1; ++i) {
        const int r0 = tile_row(i);
        uint8_t *stage = ring + st * 2 * C::kTile;
        uint64_t *bar = &s_full[warp][st];
        if (r0 <= w.rows.last) {  // (the same for the whole warp)
          if (!mbar_wait_warp(bar, phase)) {
            gave_up = true;
            break;
          }
          // `open`: every query sees every row (and, for the statistics, none is in the suffix)
          auto tile = [&](auto open_tile, int h0) {
            constexpr bool open = decltype(open_tile)::value;
            const uint8_t *sk = stage + h0 * 16 * C::kRow;
            const uint32_t k_at = smem_addr(sk), v_at = k_at + C::kTile;
            const int rh = r0 + 16 * h0;
            // ---- scores
            float raw[J][NT][4], z[J][NT][4];
#pragma unroll
            for (int h = 0; h < J; ++h) {
              uint32_t ga, gb;
              ldmatrix2(ga, gb, k_at + at2 + h * 16 * C::kRow);
              ga = __byte_perm(ga, ga, 0x3232);  // the least value twice, for three terms
              gb = __byte_perm(gb, gb, 0x3232);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_bf16(raw[h][nt], ga, gb, ga, gb, sum_12[nt], sum_3[nt], 0.f, 0.f, 0.f, 0.f);
              const uint4 pa = *(const uint4 *)(sk + (16 * h + g) * C::kRow + D / 2);
              const uint4 pb = *(const uint4 *)(sk + (16 * h + g + 8) * C::kRow + D / 2);
              const uint32_t par_a[4] = {pa.x, pa.y, pa.z, pa.w}, par_b[4] = {pb.x, pb.y, pb.z, pb.w};
#pragma unroll
              for (int j2 = 0; j2 < kPieces; j2 += 2) {
                uint32_t kw[4];
                ldmatrix4(kw, k_at + at4 + h * 16 * C::kRow + 16 * j2);
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                  const uint32_t wa = kw[2 * jj], wb = kw[2 * jj + 1], va = wa >> 8, vb = wb >> 8;
                  const uint32_t fa[4] = {wa & kQ4Low, wa & kQ4High, va & kQ4Low, va & kQ4High};
                  const uint32_t fb[4] = {wb & kQ4Low, wb & kQ4High, vb & kQ4Low, vb & kQ4High};
#pragma unroll
                  for (int gi = 0; gi < 4 / kPieces; ++gi) {
                    const int gr = (j2 + jj) * (4 / kPieces) + gi;
                    const float s_a = bf16_low(par_a[gr]), s_b = bf16_low(par_b[gr]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                      uint32_t f[4];
                      if constexpr (NT <= 2) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[e] = qf[nt][gr][e];
                      } else {
                        const uint4 v = s_q[(nt * 4 + gr) * 32 + lane];
                        f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
                      }
                      float d[4];
                      mma_bf16(d, fa[0], fb[0], fa[1], fb[1], f[0], f[1], 0.f, 0.f, 0.f, 0.f);
                      mma_bf16(d, fa[2], fb[2], fa[3], fb[3], f[2], f[3], d[0], d[1], d[2], d[3]);
                      raw[h][nt][0] = __fmaf_rn(s_a, d[0], raw[h][nt][0]);
                      raw[h][nt][1] = __fmaf_rn(s_a, d[1], raw[h][nt][1]);
                      raw[h][nt][2] = __fmaf_rn(s_b, d[2], raw[h][nt][2]);
                      raw[h][nt][3] = __fmaf_rn(s_b, d[3], raw[h][nt][3]);
                    }
                  }
                }
              }
              // in log2 units, less the maximum in use
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  z[h][nt][j] = __fmaf_rn(raw[h][nt][j], cm[nt][j & 1], -m[nt][j & 1]);
            }
            // ---- what each query may see
            if (!open) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const int last = last_seen(8 * nt + 2 * t + c), low = low_seen(last);
#pragma unroll
                  for (int h = 0; h < J; ++h)
#pragma unroll
                    for (int j = c; j < 4; j += 2) {
                      const int r = rh + 16 * h + g + 8 * (j >> 1);
                      if (hides(r, last, low)) z[h][nt][j] = kHidden;
                    }
                }
            }
            // ---- maxima, kept while no score passes them by kLazy
            float past = kHidden;
#pragma unroll
            for (int h = 0; h < J; ++h)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) past = fmaxf(past, z[h][nt][j]);
            if (__any_sync(0xffffffffu, past > kLazy)) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  // (from the sums again: a first maximum is no difference to kNone)
                  float x = m[nt][c];
#pragma unroll
                  for (int h = 0; h < J; ++h)
#pragma unroll
                    for (int j = c; j < 4; j += 2) {
                      raw[h][nt][j] = z[h][nt][j] == kHidden ? kHidden : raw[h][nt][j] * cm[nt][c];
                      x = fmaxf(x, raw[h][nt][j]);
                    }
                  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                  const float by = m[nt][c] - x, f = exp2_fast(by);
                  m[nt][c] = x;
#pragma unroll
                  for (int h = 0; h < J; ++h)
#pragma unroll
                    for (int j = c; j < 4; j += 2)
                      z[h][nt][j] = z[h][nt][j] == kHidden ? kHidden : raw[h][nt][j] - x;
                  if (STATS) {
                    top[nt][c] += by;
                    hs[nt][c] = l[nt][c] > 0.f ? f * __fmaf_rn(by, l[nt][c], hs[nt][c]) : 0.f;
                    sf[nt][c] *= f;
                  }
                  l[nt][c] *= f;
#pragma unroll
                  for (int j = c; j < 4; j += 2) {
                    ox[nt][j] *= f;
#pragma unroll
                    for (int gr = 0; gr < 4; ++gr)
#pragma unroll
                      for (int u = 0; u < 2; ++u) o[nt][gr][u][j] *= f;
                  }
                }
            }
            // ---- weights: p0 = keys 2t, 2t+1 and p1 = keys 2t+8, 2t+9 of query row g
            uint32_t p0[J][NT], p1[J][NT];
#pragma unroll
            for (int h = 0; h < J; ++h)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int c = j & 1;
                  p[j] = exp2_fast(z[h][nt][j]);
                  l[nt][c] += p[j];
                  if (STATS) {
                    top[nt][c] = fmaxf(top[nt][c], z[h][nt][j]);
                    hs[nt][c] = __fmaf_rn(p[j], z[h][nt][j], hs[nt][c]);
                  }
                }
                if (STATS && !open) {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (rh + 16 * h + g + 8 * (j >> 1) >= suffix0) sf[nt][j & 1] += p[j];
                }
                p0[h][nt] = transposed(pack_bf16(p[0], p[1]));
                p1[h][nt] = transposed(pack_bf16(p[2], p[3]));
              }
            // ---- results: this thread's keys
#pragma unroll
            for (int h = 0; h < J; ++h) {
              // half word g of the parameters of two keys: scales (g even) or least values
              uint32_t xa, xb;
              ldmatrix2_trans(xa, xb, v_at + at2 + h * 16 * C::kRow);
              uint32_t sa[4], sb[4];
#pragma unroll
              for (int gr = 0; gr < 4; ++gr) {
                sa[gr] = __shfl_sync(0xffffffffu, xa, 8 * gr + t);
                sb[gr] = __shfl_sync(0xffffffffu, xb, 8 * gr + t);
              }
              // Rows past the last hold anything, and a hidden row may hold a NaN.  Where one does: which of
              // this thread's four keys query row g of a product sees (a weight of zero does not say it: a
              // row that is seen may weigh less than the least number).
              uint32_t see0[NT], see1[NT];
              if (!open) {
                const int r = rh + 16 * h + 2 * t, e = w.rows.last;
                const bool odd =
                    finite_pair(xa, true, true) != xa || finite_pair(xb, true, true) != xb;
                xa = finite_pair(xa, r <= e, r + 1 <= e);
                xb = finite_pair(xb, r + 8 <= e, r + 9 <= e);
                const bool careful = __any_sync(0xffffffffu, odd);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  see0[nt] = see1[nt] = 0xffffffffu;
                  if (careful) {
                    const int last = last_seen(8 * nt + g), low = low_seen(last);
                    auto half = [&](int r) { return !hides(r, last, low) ? 0xffffu : 0u; };
                    see0[nt] = half(r) | half(r + 1) << 16;
                    see1[nt] = half(r + 8) | half(r + 9) << 16;
                  }
                }
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_bf16(ox[nt], xa, 0u, xb, 0u, p0[h][nt], p1[h][nt], ox[nt][0], ox[nt][1],
                         ox[nt][2], ox[nt][3]);
#pragma unroll
              for (int j2 = 0; j2 < kPieces; j2 += 2) {
                uint32_t vw[4];
                ldmatrix4_trans(vw, v_at + at4 + h * 16 * C::kRow + 16 * j2);
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                  const uint32_t wa = vw[2 * jj], wb = vw[2 * jj + 1], ua = wa >> 8, ub = wb >> 8;
                  const uint32_t fa[4] = {centred(wa & kQ4Low, false), centred(wa & kQ4High, true),
                                          centred(ua & kQ4Low, false), centred(ua & kQ4High, true)};
                  const uint32_t fb[4] = {centred(wb & kQ4Low, false), centred(wb & kQ4High, true),
                                          centred(ub & kQ4Low, false), centred(ub & kQ4High, true)};
#pragma unroll
                  for (int gi = 0; gi < 4 / kPieces; ++gi) {
                    const int gr = (j2 + jj) * (4 / kPieces) + gi;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                      const uint32_t pa = p0[h][nt], pb = p1[h][nt];
                      uint32_t b0 = mul_bf16x2(pa, sa[gr]), b1 = mul_bf16x2(pb, sb[gr]);
                      if (!open) {  // a hidden row weighs nothing, also times a NaN
                        b0 &= see0[nt];
                        b1 &= see1[nt];
                      }
#pragma unroll
                      for (int u = 0; u < 2; ++u)
                        mma_bf16(o[nt][gr][u], fa[2 * u], fa[2 * u + 1], fb[2 * u], fb[2 * u + 1], b0, b1,
                                 o[nt][gr][u][0], o[nt][gr][u][1], o[nt][gr][u][2], o[nt][gr][u][3]);
                    }
                  }
                }
              }
            }
          };
          if (r0 + kSub - 1 <= w.rows.first && r0 >= low_max && (!STATS || r0 + kSub <= suffix0)) {
#pragma unroll 1
            for (int h0 = 0; h0 < kSub / 16; h0 += J) tile(std::true_type(), h0);
          } else {
#pragma unroll 1
            for (int h0 = 0; h0 < kSub / 16; h0 += J) tile(std::false_type(), h0);
          }
          __syncwarp();  // the stage has been read
          if (lane == 0 && i + C::kStages < blk1) copy(i + C::kStages, stage, bar);
          if (++st == C::kStages) {
            st = 0;
            phase ^= 1;
          }
        }
      }
      if (gave_up && lane == 0) {
        set_status(a.status, LG_ERR_TIMEOUT);
        linger();
      }
      // every warp's copies have landed (or lingered): the ring becomes the results' place
      gave_up = __syncthreads_or(gave_up);

      // ---- the warps' results: sums of a query row over the key lanes, then over the warps
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x[4] = {m[nt][c] + (STATS ? top[nt][c] : 0.f), l[nt][c], hs[nt][c], sf[nt][c]};
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) {
            if (STATS) x[0] = fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], off));
            x[1] += __shfl_xor_sync(0xffffffffu, x[1], off);
            if (STATS) {
              x[2] += __shfl_xor_sync(0xffffffffu, x[2], off);
              x[3] += __shfl_xor_sync(0xffffffffu, x[3], off);
            }
          }
          float f = 1.f;
          if (STATS) {  // from the lagging maximum to the true one
            const float by = m[nt][c] - x[0];
            f = x[1] > 0.f ? exp2_fast(by) : 1.f;
            x[2] = x[1] > 0.f ? f * __fmaf_rn(by, x[1], x[2]) : 0.f;
            x[1] *= f;
            x[3] *= f;
          }
          const int row = 8 * nt + 2 * t + c;
          if (g == 0) s_st[warp][row] = make_float4(x[0], x[1], x[2], x[3]);
#pragma unroll
          for (int gr = 0; gr < 4; ++gr) {
            const float base = __fmaf_rn(8.f, __shfl_sync(0xffffffffu, ox[nt][c], 8 * gr + t),
                                         __shfl_sync(0xffffffffu, ox[nt][c], 8 * gr + 4 + t));
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int up = 0; up < 2; ++up)
                if (of_group<D, 8>(gr, g))
                  s_o[(warp * C::kRows + row) * (D + 1) + value_element<D>(gr, u, g, up)] =
                      f * __fmaf_rn(up ? 4.f : 64.f, o[nt][gr][u][2 * up + c], base);
          }
        }
      }
      __syncthreads();
      const bool alone = !CL && blk0 == 0 && blk1 == w.blocks.count;
      float *s_part = (float *)(smem + C::kOut);  // [row][D + 4], as in the workspace
      for (int r = warp; r < w.used; r += kWarps) {
        float mx = kNone;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) mx = fmaxf(mx, s_st[k][r].x);
        // (a part that has seen rows counts, be its factor zero: 0 x NaN)
        float f[kWarps], sl = 0.f, sh = 0.f, ss = 0.f;
        bool any[kWarps];
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float4 v = s_st[k][r];
          const float by = v.x - mx;
          any[k] = v.y != 0.f;
          f[k] = any[k] ? exp2_fast(by) : 0.f;
          sl += f[k] * v.y;
          if (STATS) {
            sh += v.y != 0.f ? f[k] * __fmaf_rn(by, v.y, v.z) : 0.f;
            ss += f[k] * v.w;
          }
        }
        const int rr = r + row_1;
        const int64_t head = ((int64_t)layer * a.T + w.off + rr / a.g) * H_q + w.kvh * a.g + rr % a.g;
        float *part = CL ? s_part + r * (D + 4) : part_row<D>(a, layer, cta, x < y0 ? 0 : 1, r);
        const float inv = sl != 0.f ? 1.f / sl : 0.f;
#pragma unroll
        for (int e = lane; e < D; e += 32) {
          float x = 0.f;
#pragma unroll
          for (int k = 0; k < kWarps; ++k)
            if (any[k]) x += f[k] * s_o[(k * C::kRows + r) * (D + 1) + e];
          if (alone)
            ((__nv_bfloat16 *)a.out)[head * D + e] = __float2bfloat16_rn(x * inv);
          else
            part[e] = x;
        }
        if (lane == 0) {
          if (!alone)
            *(float4 *)(part + D) = make_float4(mx, sl, sh, ss);
          else if (STATS)
            ((float4 *)a.stats)[head] =
                make_float4(mx * 0.6931471805599453f, sl,
                            logf(sl) - 0.6931471805599453f * sh * inv, ss * inv);
        }
      }
      if constexpr (CL) {
        // the cluster's results: a warp 32 elements of a row, lane k the k-th CTA's statistics
        cg::cluster_group cl = cg::this_cluster();
        __shared__ int s_no;
        if (tid == 0) s_no = bad || gave_up;
        cl.sync();
        bool no = false;
        for (int k = 0; k < a.cluster; ++k) no |= *cl.map_shared_rank(&s_no, k) != 0;
        const int n = no ? 0 : w.used * (D / 32);
        for (int i = (int)cl.block_rank() * kWarps + warp; i < n; i += a.cluster * kWarps) {
          const int r = i / (D / 32), e = i % (D / 32) * 32 + lane;
          const float4 v = *(const float4 *)(cl.map_shared_rank(s_part, lane % a.cluster) + r * (D + 4) + D);
          const bool any = v.y != 0.f;
          const unsigned seen = __ballot_sync(0xffffffffu, any);
          const float mx = warp_max(any ? v.x : kNone), by = v.x - mx;
          const float f = any ? exp2_fast(by) : 0.f;
          float sl = f * v.y, sh = any ? f * __fmaf_rn(by, v.y, v.z) : 0.f, ss = f * v.w;
#pragma unroll
          for (int o = 1; o < kClusterMost; o <<= 1) {
            if (o >= a.cluster) break;
            sl += __shfl_xor_sync(0xffffffffu, sl, o);
            sh += __shfl_xor_sync(0xffffffffu, sh, o);
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
          }
          float y = 0.f;
#pragma unroll
          for (int k = 0; k < kClusterMost; ++k) {
            if (k >= a.cluster) break;
            const float fk = __shfl_sync(0xffffffffu, f, k);
            const float z = cl.map_shared_rank(s_part, k)[r * (D + 4) + e];
            if (seen >> k & 1) y += fk * z;
          }
          const float inv = sl != 0.f ? 1.f / sl : 0.f;
          const int rr = r + row_1;
          const int64_t head = ((int64_t)layer * a.T + w.off + rr / a.g) * H_q + w.kvh * a.g + rr % a.g;
          ((__nv_bfloat16 *)a.out)[head * D + e] = __float2bfloat16_rn(y * inv);
          if (STATS && e == 0)
            ((float4 *)a.stats)[head] = make_float4(mx * 0.6931471805599453f, sl,
                                                    logf(sl) - 0.6931471805599453f * sh * inv, ss * inv);
        }
        cl.sync();  // read before a CTA ends
        return;
      }
      fence_proxy_async_smem();
      __syncthreads();  // the results have been read: the ring is the next piece's
    }
    // the next item
    if (++w.tile == tiles) {
      w.tile = 0;
      if (++w.kvh == a.H_kv) {
        w.kvh = 0;
        if (x + units >= y1) break;
        do q4_seq(a, ++seq, w.q, w.off);
        while (w.q.m == 0);
        // (x is the old sequence's last item: the loop adds its units)
        x += units;
        units = q4_units(w.q, a.shape);
        x -= units;
        tiles = q4_tiles(w.q, a.shape);
      }
    }
  }
}

// The CTAs' results of a cut item (blockIdx = (the CTA whose start cuts it, 16 rows, layer)): the
// warps share out the rows, then the parts of a row.  The maximum of all parts comes first, a lane
// a part, then their sums with nothing but additions between the loads.
constexpr int kMergeWarps = 16;

template <int D, bool STATS>
__global__ void __launch_bounds__(32 * kMergeWarps) q4_merge_kernel(Q4AttendArgs a) {
  constexpr int kE = D / 32;
  __shared__ float s_x[kMergeWarps][D];
  __shared__ float4 s_v[kMergeWarps];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int layer = blockIdx.z, r0 = blockIdx.y * kMergeWarps;
  pdl_enter();
  const Q4Cut w = *cut_at(a, D, layer, blockIdx.x);
  if (tid == 0) s_bad = status_bad(a.status);
  __syncthreads();
  if (s_bad) return;
  if (STATS && r0 == 0) {  // empty sequences attend to nothing
    const int H_q = a.H_kv * a.g;
    for (int b = blockIdx.x; b < a.batch; b += a.ctas) {
      if (a.len[b] != 0) continue;
      const int64_t head = ((int64_t)layer * a.T + b) * H_q;
      for (int e = tid; e < H_q * D / 2; e += 32 * kMergeWarps) ((uint32_t *)a.out)[head * D / 2 + e] = 0u;
      for (int h = tid; h < H_q; h += 32 * kMergeWarps)
        ((float4 *)a.stats)[head + h] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
  }
  if (w.step == 0 || r0 >= w.used) return;
  const int c0 = blockIdx.x - 1;  // the CTA that the item began in
  auto cut = [&](int c) { return q4_cut(c * w.step - w.x0, w.count); };  // blocks before CTA c
  // where one part has every block, its CTA wrote the result
  int p0 = 0, p1 = (int)plan_div(w.x0 + w.units - 1, w.step) + 1 - c0;  // the parts with blocks
  while (cut(c0 + p0 + 1) == 0) ++p0;
  while (cut(c0 + p1 - 1) == w.count) --p1;
  if (p1 - p0 == 1) return;
  int share2 = 0;  // log2 of the warps of a row
  while (min(w.used - r0, kMergeWarps) << (share2 + 1) <= kMergeWarps) ++share2;
  const int r = r0 + (warp >> share2), sub = warp & ((1 << share2) - 1);
  float mx = kNone, sl = 0.f, sh = 0.f, ss = 0.f, x[kE] = {};
  if (r < w.used) {
    auto part_of = [&](int k) { return part_row<D>(a, layer, c0 + k, k == 0, r); };
    for (int c = p0 + lane; c < p1; c += 32) mx = fmaxf(mx, part_of(c)[D]);
    mx = warp_max(mx);
#pragma unroll 4
    for (int c = p0 + sub; c < p1; c += 1 << share2) {
      const float *part = part_of(c);
      const float4 v = *(const float4 *)(part + D);
      float y[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) y[e] = part[lane + 32 * e];
      const bool any = v.y != 0.f;
      const float by = v.x - mx, f = any ? exp2_fast(by) : 0.f;
      sl += f * v.y;
      if (STATS) {
        sh += any ? f * __fmaf_rn(by, v.y, v.z) : 0.f;
        ss += f * v.w;
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) x[e] += any ? f * y[e] : 0.f;
    }
  }
  if (share2) {
#pragma unroll
    for (int e = 0; e < kE; ++e) s_x[warp][lane + 32 * e] = x[e];
    if (lane == 0) s_v[warp] = make_float4(0.f, sl, sh, ss);
    __syncthreads();
    if (sub) return;
    for (int k = 1; k < 1 << share2; ++k) {
      const float4 v = s_v[warp + k];
      sl += v.y;
      sh += v.z;
      ss += v.w;
#pragma unroll
      for (int e = 0; e < kE; ++e) x[e] += s_x[warp + k][lane + 32 * e];
    }
  }
  if (r >= w.used) return;
  const float inv = sl != 0.f ? 1.f / sl : 0.f;
  const int rr = r + w.row_1, H_q = a.H_kv * a.g;
  const int64_t head = w.head + (int64_t)(rr / a.g) * H_q + rr % a.g;
#pragma unroll
  for (int e = 0; e < kE; ++e)
    ((__nv_bfloat16 *)a.out)[head * D + 32 * e + lane] = __float2bfloat16_rn(x[e] * inv);
  if (STATS && lane == 0)
    ((float4 *)a.stats)[head] = make_float4(mx * 0.6931471805599453f, sl,
                                            logf(sl) - 0.6931471805599453f * sh * inv, ss * inv);
}

template <int D, int NT, bool STATS, bool CL>
cudaError_t launch_as(const Q4AttendArgs &a, cudaStream_t s) {
  using C = Q4Cfg<D, NT>;
  if constexpr (C::kSmem > 44 * 1024)  // (48 KB with the static arrays need no leave)
    LG_TRY(cudaFuncSetAttribute(q4_attend_kernel<D, NT, STATS, CL>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.ctas, a.n_layers);
  cfg.blockDim = kThreads;
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, q4_attend_kernel<D, NT, STATS, CL>, a);
}

template <int D, int NT, bool STATS>
cudaError_t launch_nt(const Q4AttendArgs &a, cudaStream_t s) {
  return a.cluster ? launch_as<D, NT, STATS, true>(a, s) : launch_as<D, NT, STATS, false>(a, s);
}

template <int D, bool STATS>
cudaError_t launch_d(const Q4AttendArgs &a, cudaStream_t s) {
  switch (a.shape.rows) {
    case 8: LG_TRY((launch_nt<D, 1, STATS>(a, s))); break;
    case 16: if constexpr (!STATS) LG_TRY((launch_nt<D, 2, STATS>(a, s))); break;
    case 24: if constexpr (!STATS) LG_TRY((launch_nt<D, 3, STATS>(a, s))); break;
    default: if constexpr (!STATS) LG_TRY((launch_nt<D, 4, STATS>(a, s))); break;
  }
  if (!a.cluster)
    LG_TRY(launch_pdl(q4_merge_kernel<D, STATS>,
                      dim3(a.ctas, (a.shape.rows + kMergeWarps - 1) / kMergeWarps, a.n_layers),
                      32 * kMergeWarps, 0, s, a));
  return cudaGetLastError();
}

}  // namespace

Q4Grid q4_grid(int n_layers, int batch, int H_kv, int g, int d, int max_new, int max_len, int window,
               int sink) {
  Q4Grid r;
  // (a step in which every sequence rests, of no new rows, has a size too)
  const int64_t rows = plan_max(1, max_new) * g;
  r.rows = rows >= 32 ? 32 : (int)((rows + 7) / 8 * 8);
  const int64_t tiles = (rows + r.rows - 1) / r.rows;
  const int64_t blocks = ((int64_t)max_len + (1 << kBn2) - 1) >> kBn2;
  // What the 152 SMs of a GB300 hold at once, over the layers, rounded down: all shares are equal, so
  // CTAs past that are a second wave (28 layers of 64 sequences of up to 4096 rows: 476 CTAs 919 us, 448
  // 643; 64 layers of up to 2048: 512 and 448, 1212 and 869; one layer is 456 either way).  No more than
  // there are blocks.
  const int64_t fit = 152 * (r.rows <= 8 ? 3 : 2);
  const int64_t most = (int64_t)batch * H_kv * tiles * (blocks + kQ4ItemUnits);
  r.ctas = (int)plan_max(1, plan_min(most, fit / n_layers));
  r.part_bytes = (size_t)n_layers * r.ctas * (2 * r.rows * (d + 4) * sizeof(float) + sizeof(Q4Cut));
  r.part_bytes = (r.part_bytes + 255) / 256 * 256;
  // Few items of few blocks: as many CTAs each as the GPU holds of them, up to eight, which join
  // their results themselves; while a CTA has at most 16 blocks of eight query rows, or 5 of more.
  // (us in a line with its second kernel and in clusters, 8 kv-heads: one sequence of 1025 rows
  // 11.2 and 7.8, 24 of 700 17.0 and 11.8, 24 of 2049 22.8 and 19.6; with 16 query rows 12 of 1500
  // 16.0 and, at 6 blocks a CTA, 18.4.)
  const int64_t items = (int64_t)batch * H_kv * tiles;
  const Q4Shape shape{r.rows, g, window, sink, H_kv};
  const int one = q4_units(ChunkSeq{max_len, max_new < max_len ? max_new : max_len}, shape) - kQ4ItemUnits;
  r.cluster = 0;
  for (int n = kClusterMost; n >= 1 && !r.cluster; n /= 2)
    if (items * n_layers * n <= fit && one <= n * (r.rows <= 8 ? 16 : 5)) r.cluster = n;
  if (r.cluster) r.ctas = (int)items * r.cluster;
  return r;
}

cudaError_t launch_q4_attend(const Q4AttendArgs &a, int d, cudaStream_t s) {
  if (a.stats) return d == 128 ? launch_d<128, true>(a, s) : launch_d<64, true>(a, s);
  return d == 128 ? launch_d<128, false>(a, s) : launch_d<64, false>(a, s);
}

}  // namespace lg
