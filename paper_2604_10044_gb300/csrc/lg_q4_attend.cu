// Attention of few query rows of a kv-head (a token, or some drafted tokens, a sequence) over a 4-bit
// cache, with the statistics that the guard reads of a single token.
//
// A warp takes 16 rows of keys and values at a time through mma.sync (M = 16 keys or 16 elements, N = 8
// query rows, K = 16), and no value is ever formed from its code:
//   scores   q . k = sum over groups of (s_g sum_e q_e c_e) + sum_g lo_g sum_{e in g} q_e.  The codes enter
//            as the bf16 numbers 128 + c (a shift and a mask and an or for two), the products of a group
//            start from -128 sum q instead of zero, and the four sums are joined by the rows' scales in
//            fp32.  The least values are one more product, with sums of q in two bf16 terms.  q and the
//            codes are exact, so are the products.
//   results  sum_k p_k v_k = sum_k (p_k s_kg)(c - 8) + sum_k p_k (lo_kg + 8 s_kg): for each group the weights
//            times its scales, rounded to bf16, are the second operand, and one more product takes the
//            groups' middles.  Codes about zero, not 128 + c with the 128 taken off at the end: sums then
//            stay small beside what the matrix unit drops of them (over 262143 rows of independent values
//            the result was off by 1.5 % with 128), and a weight's second rounding meets |c - 8|, not c.
// A row's pair of codes for the results is a pair of keys: two rows' half words joined by one byte
// permutation, then the same shift and mask.
//
// Weights are 2^(z - m) with a maximum m that may lag: it is formed anew only when a score passes it
// by 8, so a tile asks one vote.  Every warp has its own m and sums; the CTA's four are merged at its
// end, and the CTAs of an item by a second kernel.
//
// Every warp copies its own 16 rows a block (bulk copies into a ring of its own), so warps never wait
// for one another.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lg_chunk_plan.cuh"
#include "lg_q4.cuh"

namespace lg {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kSub = 16;             // rows of a warp's tile
constexpr int kBn2 = 6;              // log2 of a CTA's block: kWarps tiles
constexpr int kBn = 1 << kBn2;
constexpr float kLazy = 8.f;         // log2 units that a weight may pass 1 by
constexpr float kHidden = -1e38f;    // score of a row that a query does not see
constexpr float kNone = -1e30f;      // maximum of a query that has seen nothing
static_assert(kWarps * kSub == kBn, "a tile a warp");

template <int D, int NT>
struct Q4Cfg {
  static constexpr int kRow = q4_row_bytes(D);
  static constexpr int kTile = kSub * kRow;         // of keys, or of values
  static constexpr int kStages = 4;
  static constexpr int kRing = kWarps * kStages * 2 * kTile;
  static constexpr int kRows = 8 * NT;
  static constexpr int kOut = kWarps * kRows * (D + 1) * 4;  // the warps' results, for their merge
  static constexpr int kQ = NT > 2 ? NT * 4 * 32 * 16 : 0;   // fragments of q, unless in registers
  static constexpr int kSmem = (kRing > kOut ? kRing : kOut) + kQ;
};

// A group's second operands of the scores for thread t, from a query row (null: zeros): slots 2t, 2t+1
// and 2t+8, 2t+9 of each product hold the elements that q4_pair leaves of the thread's codes.
template <int D>
__device__ __forceinline__ void query_fragment(const __nv_bfloat16 *q, int gr, int t,
                                               uint32_t (&f)[D / 32]) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if constexpr (D == 128) {  // one word of codes a row: its eight elements in order
    if (q) v = *(const uint4 *)(q + 8 * (4 * gr + t));
    f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
  } else {  // half a word: the even elements or the odd ones
    if (q) v = *(const uint4 *)(q + 8 * (2 * gr + (t >> 1)));
    const uint32_t sel = t & 1 ? 0x7632 : 0x5410;
    f[0] = __byte_perm(v.x, v.y, sel);
    f[1] = __byte_perm(v.z, v.w, sel);
  }
}

// the element of row r (g or g + 8) of result tile u of group gr
template <int D>
__device__ __forceinline__ int value_element(int gr, int u, int r) {
  const int g = r & 7, up = r >> 3;
  if constexpr (D == 128) {
    return 8 * (4 * gr + (g >> 1)) + 2 * (2 * u + up) + (g & 1);
  } else {
    const int n = 2 * (g & 3) + up;  // nibble of the word
    return 8 * (2 * gr + (g >> 2)) + (n < 4 ? 2 * n : 2 * (n - 4) + 1);
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t *)&h;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
  return *(const uint32_t *)&r;
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hsub2(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
  return *(const uint32_t *)&r;
}

constexpr uint32_t k136 = 0x43084308u;  // two bf16 numbers 136: 128 + c less 136 is c - 8, exactly

// lo + 8 s of a group of two rows, rounded once
__device__ __forceinline__ uint32_t middles(uint32_t par0, uint32_t par1) {
  const uint32_t s = __byte_perm(par0, par1, 0x5410), lo = __byte_perm(par0, par1, 0x7632);
  const uint32_t eight = 0x41004100u;
  const __nv_bfloat162 r = __hfma2(*(const __nv_bfloat162 *)&s, *(const __nv_bfloat162 *)&eight,
                                   *(const __nv_bfloat162 *)&lo);
  return *(const uint32_t *)&r;
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// a partial result: [rows][D + 4], the sums and {m, l, sum p (z - m), suffix}; m the true maximum
template <int D>
__device__ __forceinline__ float *part_row(const Q4AttendArgs &a, int64_t item, int chunk, int r) {
  return a.part + ((item * a.chunks + chunk) * a.rows + r) * (int64_t)(D + 4);
}

struct Q4Item {
  int layer, b, kvh, tile, off;
  ChunkSeq q;
  TileRows rows;
  TileBlocks blocks;
  int used;  // query rows
};

// item number -> what it is; false for one without queries, or a length out of bounds (recorded)
__device__ __forceinline__ bool q4_item(const Q4AttendArgs &a, int64_t item, Q4Item &w) {
  w.tile = (int)(item % a.tiles);
  item /= a.tiles;
  w.kvh = (int)(item % a.H_kv);
  item /= a.H_kv;
  w.b = (int)(item % a.batch);
  w.layer = a.layer0 + (int)(item / a.batch);
  w.q.n = a.len[w.b];
  w.off = a.off ? a.off[w.b] : w.b;
  w.q.m = a.off ? a.off[w.b + 1] - w.off : (w.q.n > 0 ? 1 : 0);
  if (w.q.n < 0 || w.q.n > a.max_len || w.q.m < 0 || w.q.m > a.max_new || w.q.m > w.q.n ||
      w.off < 0 || w.off + w.q.m > a.T) {
    if (threadIdx.x == 0) set_status(a.status, LG_ERR_CAPACITY);
    return false;
  }
  w.used = min(a.rows, w.q.m * a.g - w.tile * a.rows);
  if (w.used <= 0) return false;
  // the rows that its first and last query see
  const int t0 = w.tile * a.rows / a.g, t1 = (w.tile * a.rows + w.used - 1) / a.g;
  w.rows.first = w.q.n - w.q.m + t0;
  w.rows.last = w.q.n - w.q.m + t1;
  w.rows.lo = a.window ? (int)plan_max(0, (int64_t)w.rows.first + 1 - a.window) : 0;
  w.rows.sinks = min(a.sink, w.rows.lo);
  w.blocks = tile_blocks(w.rows, kBn2);
  return true;
}

template <int D, int NT, bool STATS>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 4 : NT == 2 ? 3 : 2) q4_attend_kernel(Q4AttendArgs a) {
  using C = Q4Cfg<D, NT>;
  constexpr int kMpg = D == 128 ? 2 : 1;  // products of a group
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
  if (cta_status_bad(a.status)) return;
  const int64_t item = blockIdx.x / a.chunks;
  const int chunk = blockIdx.x % a.chunks;
  Q4Item w;
  if (!q4_item(a, item, w)) {
    if (STATS && w.q.n == 0 && chunk == 0) {  // an empty sequence attends to nothing
      const int64_t head = (((int64_t)w.layer - a.layer0) * a.T + w.off) * a.H_kv * a.g + w.kvh * a.g;
      for (int e = tid; e < a.g * D / 2; e += kThreads) ((uint32_t *)a.out)[head * D / 2 + e] = 0u;
      if (tid < a.g) ((float4 *)a.stats)[head + tid] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
    return;
  }
  const int blk0 = chunk * a.blocks, blk1 = min(blk0 + a.blocks, w.blocks.count);
  if (blk0 >= blk1) return;

  // this warp's copies: its 16 rows of each block
  uint8_t *ring = smem + warp * C::kStages * 2 * C::kTile;
  const int64_t row0 = ((int64_t)w.layer * a.H_kv + w.kvh) * a.S_total + a.seq_off[w.b];
  const uint8_t *gk = a.K + row0 * C::kRow, *gv = a.V + row0 * C::kRow;
  auto tile_row = [&](int i) { return (w.blocks.index(i) << kBn2) + warp * kSub; };
  auto copy = [&](int i) {  // lane 0: block i into its stage
    const int r = tile_row(i);
    const int n = min(kSub, w.rows.last + 1 - r);
    if (n <= 0) return;
    const int st = (i - blk0) % C::kStages;
    uint8_t *to = ring + st * 2 * C::kTile;
    mbar_arrive_expect_tx(&s_full[warp][st], 2 * n * C::kRow);
    bulk_load(to, gk + (int64_t)r * C::kRow, n * C::kRow, &s_full[warp][st]);
    bulk_load(to + C::kTile, gv + (int64_t)r * C::kRow, n * C::kRow, &s_full[warp][st]);
  };
  if (lane == 0)
    for (int i = blk0; i < min(blk1, blk0 + C::kStages); ++i) copy(i);

  // q as second operands, -128 times its groups' sums, and the sums in two terms for the least values
  const int H_q = a.H_kv * a.g;
  const __nv_bfloat16 *q = (const __nv_bfloat16 *)a.q +
                           (((int64_t)w.layer - a.layer0) * a.T + w.off) * H_q * D +
                           (int64_t)w.kvh * a.g * D;
  auto q_row = [&](int r) {  // row r of the item, or null
    r += w.tile * a.rows;
    return r < w.tile * a.rows + w.used ? q + ((int64_t)(r / a.g) * H_q + r % a.g) * D : nullptr;
  };
  uint32_t qf[NT <= 2 ? NT : 1][4][2 * kMpg];
  uint4 *s_q = (uint4 *)(smem + C::kSmem - C::kQ);
  float init[NT][4][2];   // [group][column 2t, 2t+1]
  uint32_t sum_hi[NT], sum_lo[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const __nv_bfloat16 *src = q_row(8 * nt + g);
    float mine = 0.f;
#pragma unroll
    for (int gr = 0; gr < 4; ++gr) {
      uint32_t f[2 * kMpg];
      query_fragment<D>(src, gr, t, f);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * kMpg; ++i) sum += bf16_low(f[i]) + bf16_high(f[i]);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (t == gr) mine = sum;
      // columns 2t, 2t+1 of the scores belong to the query rows of lanes 8t and 8t + 4
      init[nt][gr][0] = -128.f * __shfl_sync(0xffffffffu, sum, 8 * t);
      init[nt][gr][1] = -128.f * __shfl_sync(0xffffffffu, sum, 8 * t + 4);
      if constexpr (NT <= 2) {
#pragma unroll
        for (int i = 0; i < 2 * kMpg; ++i) qf[nt][gr][i] = f[i];
      } else if (warp == 0) {
        s_q[(nt * 4 + gr) * 32 + lane] =
            make_uint4(f[0], f[1], kMpg == 2 ? f[2 * kMpg - 2] : 0u, kMpg == 2 ? f[2 * kMpg - 1] : 0u);
      }
    }
    const float hi = __bfloat162float(__float2bfloat16_rn(mine));
    sum_hi[nt] = pack_bf16(0.f, hi);
    sum_lo[nt] = pack_bf16(0.f, mine - hi);
  }
  if constexpr (NT > 2) __syncthreads();

  const int low_max = a.window ? (int)plan_max(0, (int64_t)w.rows.last + 1 - a.window) : 0;
  const int suffix0 = w.q.n - a.suffix_w;  // (n and suffix_w are positive)

  float o[NT][4][kMpg][4] = {};
  float ox[NT][4] = {};  // rows gr: the weights times the middles of group gr
  float m[NT][2], top[NT][2], l[NT][2], hs[NT][2], sf[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      m[nt][c] = top[nt][c] = kNone;
      l[nt][c] = hs[nt][c] = sf[nt][c] = 0.f;
    }

  bool gave_up = false;
  for (int i = blk0; i < blk1; ++i) {
    const int r0 = tile_row(i);
    const int st = (i - blk0) % C::kStages;
    if (r0 <= w.rows.last) {  // (the same for the whole warp)
      if (!mbar_wait_warp(&s_full[warp][st], ((i - blk0) / C::kStages) & 1)) {
        gave_up = true;
        break;
      }
      const uint8_t *sk = ring + st * 2 * C::kTile, *sv = sk + C::kTile;
      // ---- scores
      float z[NT][4];
      {
        const uint8_t *ka = sk + g * C::kRow, *kb = ka + 8 * C::kRow;
        const uint4 pa = *(const uint4 *)(ka + D / 2), pb = *(const uint4 *)(kb + D / 2);
        const uint32_t ga = *(const uint32_t *)(ka + D / 2 + 4 * t);
        const uint32_t gb = *(const uint32_t *)(kb + D / 2 + 4 * t);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          mma_bf16(z[nt], ga & 0xffff0000u, gb & 0xffff0000u, ga & 0xffff0000u, gb & 0xffff0000u,
                   sum_hi[nt], sum_lo[nt], 0.f, 0.f, 0.f, 0.f);
        const uint32_t par_a[4] = {pa.x, pa.y, pa.z, pa.w}, par_b[4] = {pb.x, pb.y, pb.z, pb.w};
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
          uint32_t wa, wb;
          if constexpr (D == 128) {
            wa = *(const uint32_t *)(ka + 16 * gr + 4 * t);
            wb = *(const uint32_t *)(kb + 16 * gr + 4 * t);
          } else {
            wa = *(const uint16_t *)(ka + 8 * gr + 2 * t);
            wb = *(const uint16_t *)(kb + 8 * gr + 2 * t);
            wa |= wa << 12;
            wb |= wb << 12;
          }
          constexpr int kStep = D == 128 ? 4 : 8;
          uint32_t fa[2 * kMpg], fb[2 * kMpg];
#pragma unroll
          for (int j = 0; j < 2 * kMpg; ++j) {
            fa[j] = q4_pair(wa >> (kStep * j));
            fb[j] = q4_pair(wb >> (kStep * j));
          }
          const float s_a = bf16_low(par_a[gr]), s_b = bf16_low(par_b[gr]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint32_t f[2 * kMpg];
            if constexpr (NT <= 2) {
#pragma unroll
              for (int j = 0; j < 2 * kMpg; ++j) f[j] = qf[nt][gr][j];
            } else {
              const uint4 v = s_q[(nt * 4 + gr) * 32 + lane];
              f[0] = v.x;
              f[1] = v.y;
              if constexpr (kMpg == 2) f[2] = v.z, f[3] = v.w;
            }
            float d[4];
            mma_bf16(d, fa[0], fb[0], fa[1], fb[1], f[0], f[1], init[nt][gr][0], init[nt][gr][1],
                     init[nt][gr][0], init[nt][gr][1]);
            if constexpr (kMpg == 2)
              mma_bf16(d, fa[2], fb[2], fa[3], fb[3], f[2], f[3], d[0], d[1], d[2], d[3]);
            z[nt][0] = __fmaf_rn(s_a, d[0], z[nt][0]);
            z[nt][1] = __fmaf_rn(s_a, d[1], z[nt][1]);
            z[nt][2] = __fmaf_rn(s_b, d[2], z[nt][2]);
            z[nt][3] = __fmaf_rn(s_b, d[3], z[nt][3]);
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[nt][j] *= a.qscale;
      // ---- what each query may see
      const bool open = r0 + kSub - 1 <= w.rows.first && r0 >= low_max;
      if (!open) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int qr = min(8 * nt + 2 * t + c, w.used - 1) + w.tile * a.rows;
            const int last = w.q.n - w.q.m + qr / a.g;  // the query's own row
            const int low = a.window ? (int)plan_max(0, (int64_t)last + 1 - a.window) : 0;
#pragma unroll
            for (int j = c; j < 4; j += 2) {
              const int r = r0 + g + 8 * (j >> 1);
              if (r > last || (r < low && r >= a.sink)) z[nt][j] = kHidden;
            }
          }
      }
      // ---- maxima, kept while no score passes them by kLazy
      bool past = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) past |= z[nt][j] > m[nt][j & 1] + kLazy;
      if (__any_sync(0xffffffffu, past)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = fmaxf(fmaxf(z[nt][c], z[nt][2 + c]), m[nt][c]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float by = m[nt][c] - x, f = exp2_fast(by);
            m[nt][c] = x;
            if (STATS) hs[nt][c] = l[nt][c] > 0.f ? f * __fmaf_rn(by, l[nt][c], hs[nt][c]) : 0.f;
            l[nt][c] *= f;
            if (STATS) sf[nt][c] *= f;
#pragma unroll
            for (int j = c; j < 4; j += 2) {
              ox[nt][j] *= f;
#pragma unroll
              for (int gr = 0; gr < 4; ++gr)
#pragma unroll
                for (int u = 0; u < kMpg; ++u) o[nt][gr][u][j] *= f;
            }
          }
      }
      // ---- weights: b0 = keys 2t, 2t+1 and b1 = keys 2t+8, 2t+9 of query row g
      uint32_t p0[NT], p1[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = j & 1;
          const float d = z[nt][j] - m[nt][c];
          p[j] = exp2_fast(d);
          l[nt][c] += p[j];
          if (STATS) {
            top[nt][c] = fmaxf(top[nt][c], z[nt][j]);
            hs[nt][c] = __fmaf_rn(p[j], d, hs[nt][c]);
          }
        }
        if (STATS && r0 + kSub > suffix0) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (r0 + g + 8 * (j >> 1) >= suffix0) sf[nt][j & 1] += p[j];
        }
        p0[nt] = transposed(pack_bf16(p[0], p[1]));
        p1[nt] = transposed(pack_bf16(p[2], p[3]));
      }
      // ---- results: this thread's keys
      {
        const uint8_t *v0 = sv + (2 * t) * C::kRow, *v1 = v0 + C::kRow, *v2 = v0 + 8 * C::kRow,
                      *v3 = v0 + 9 * C::kRow;
        const int lw = D / 2 + 4 * (g & 3);
        uint32_t l0 = *(const uint32_t *)(v0 + lw), l1 = *(const uint32_t *)(v1 + lw);
        uint32_t l2 = *(const uint32_t *)(v2 + lw), l3 = *(const uint32_t *)(v3 + lw);
        if (!open) {  // rows past the last hold anything, and a hidden row may hold a NaN
          const int r = r0 + 2 * t, e = w.rows.last;
          l0 = r > e || (l0 & 0x7f80u) == 0x7f80u ? 0u : l0;
          l1 = r + 1 > e || (l1 & 0x7f80u) == 0x7f80u ? 0u : l1;
          l2 = r + 8 > e || (l2 & 0x7f80u) == 0x7f80u ? 0u : l2;
          l3 = r + 9 > e || (l3 & 0x7f80u) == 0x7f80u ? 0u : l3;
        }
        const uint32_t la = middles(l0, l1), lb = middles(l2, l3);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          mma_bf16(ox[nt], la, la, lb, lb, p0[nt], p1[nt], ox[nt][0], ox[nt][1], ox[nt][2],
                   ox[nt][3]);
        const uint4 s0 = *(const uint4 *)(v0 + D / 2), s1 = *(const uint4 *)(v1 + D / 2);
        const uint4 s2 = *(const uint4 *)(v2 + D / 2), s3 = *(const uint4 *)(v3 + D / 2);
        const uint32_t sa[4] = {__byte_perm(s0.x, s1.x, 0x5410), __byte_perm(s0.y, s1.y, 0x5410),
                                __byte_perm(s0.z, s1.z, 0x5410), __byte_perm(s0.w, s1.w, 0x5410)};
        const uint32_t sb[4] = {__byte_perm(s2.x, s3.x, 0x5410), __byte_perm(s2.y, s3.y, 0x5410),
                                __byte_perm(s2.z, s3.z, 0x5410), __byte_perm(s2.w, s3.w, 0x5410)};
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
          uint32_t xa, xb;
          if constexpr (D == 128) {
            const int at = 16 * gr + 2 * g;
            xa = *(const uint16_t *)(v0 + at) | (uint32_t)*(const uint16_t *)(v1 + at) << 16;
            xb = *(const uint16_t *)(v2 + at) | (uint32_t)*(const uint16_t *)(v3 + at) << 16;
          } else {
            const int at = 8 * gr + g;
            xa = v0[at] | (uint32_t)v1[at] << 16;
            xb = v2[at] | (uint32_t)v3[at] << 16;
          }
          uint32_t fa[2 * kMpg], fb[2 * kMpg];
#pragma unroll
          for (int j = 0; j < 2 * kMpg; ++j) {
            fa[j] = sub_bf16x2(q4_pair(xa >> (4 * j)), k136);
            fb[j] = sub_bf16x2(q4_pair(xb >> (4 * j)), k136);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint32_t b0 = mul_bf16x2(p0[nt], sa[gr]), b1 = mul_bf16x2(p1[nt], sb[gr]);
            if (!open) {  // a weight of zero stays zero, whatever the scale holds
              b0 &= (p0[nt] & 0xffffu ? 0xffffu : 0u) | (p0[nt] >> 16 ? 0xffff0000u : 0u);
              b1 &= (p1[nt] & 0xffffu ? 0xffffu : 0u) | (p1[nt] >> 16 ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int u = 0; u < kMpg; ++u)
              mma_bf16(o[nt][gr][u], fa[2 * u], fa[2 * u + 1], fb[2 * u], fb[2 * u + 1], b0, b1,
                       o[nt][gr][u][0], o[nt][gr][u][1], o[nt][gr][u][2], o[nt][gr][u][3]);
          }
        }
      }
    }
    __syncwarp();  // the stage has been read
    if (lane == 0 && i + C::kStages < blk1) copy(i + C::kStages);
  }
  if (gave_up && lane == 0) {
    set_status(a.status, LG_ERR_TIMEOUT);
    linger();
  }
  // every warp's copies have landed (or lingered): the ring becomes the results' place
  __syncthreads();

  // ---- the warps' results: sums of a query row over the key lanes, then over the warps
  float *s_o = (float *)smem;                     // [warp][row][D + 1]
  __shared__ float4 s_st[kWarps][8 * NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float x[4] = {STATS ? top[nt][c] : m[nt][c], l[nt][c], hs[nt][c], sf[nt][c]};
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
        const float base = __shfl_sync(0xffffffffu, ox[nt][c], 4 * gr + t);
#pragma unroll
        for (int u = 0; u < kMpg; ++u)
#pragma unroll
          for (int up = 0; up < 2; ++up)
            s_o[(warp * C::kRows + row) * (D + 1) + value_element<D>(gr, u, g + 8 * up)] =
                f * (o[nt][gr][u][2 * up + c] + base);
      }
    }
  }
  __syncthreads();
  const bool alone = a.chunks == 1 || (chunk == 0 && w.blocks.count <= a.blocks);
  for (int r = warp; r < w.used; r += kWarps) {
    float mx = kNone;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) mx = fmaxf(mx, s_st[k][r].x);
    float f[kWarps], sl = 0.f, sh = 0.f, ss = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float4 v = s_st[k][r];
      const float by = v.x - mx;
      f[k] = v.y != 0.f ? exp2_fast(by) : 0.f;
      sl += f[k] * v.y;
      if (STATS) {
        sh += v.y != 0.f ? f[k] * __fmaf_rn(by, v.y, v.z) : 0.f;
        ss += f[k] * v.w;
      }
    }
    const int rr = r + w.tile * a.rows;
    const int64_t head = (((int64_t)w.layer - a.layer0) * a.T + w.off + rr / a.g) * H_q +
                         w.kvh * a.g + rr % a.g;
    float *part = part_row<D>(a, item, chunk, r);
    const float inv = sl != 0.f ? 1.f / sl : 0.f;
#pragma unroll
    for (int e = lane; e < D; e += 32) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k)
        if (f[k] != 0.f) x += f[k] * s_o[(k * C::kRows + r) * (D + 1) + e];
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
}

// The CTAs' results of an item's row, a warp a row, four elements (two) a lane.
template <int D, bool STATS>
__global__ void __launch_bounds__(kThreads) q4_merge_kernel(Q4AttendArgs a) {
  pdl_enter();
  if (cta_status_bad(a.status)) return;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t item = row / a.rows;
  const int r = (int)(row % a.rows);
  if (item >= (int64_t)a.n_layers * a.batch * a.H_kv * a.tiles) return;
  Q4Item w;
  if (!q4_item(a, item, w)) return;
  const int H_q = a.H_kv * a.g;
  if (r >= w.used || w.blocks.count <= a.blocks) return;
  const int parts = (w.blocks.count + a.blocks - 1) / a.blocks;
  float mx = kNone, sl = 0.f, sh = 0.f, ss = 0.f, x[D / 32] = {};
#pragma unroll 4
  for (int c = 0; c < parts; ++c) {
    const float *part = part_row<D>(a, item, c, r);
    const float4 v = *(const float4 *)(part + D);
    float y[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) y[e] = part[lane + 32 * e];
    if (v.y == 0.f) continue;
    const float up = fmaxf(mx, v.x), by0 = mx - up, by1 = v.x - up;
    const float f0 = exp2_fast(by0), f1 = exp2_fast(by1);
    if (STATS) {
      sh = (sl != 0.f ? f0 * __fmaf_rn(by0, sl, sh) : 0.f) + f1 * __fmaf_rn(by1, v.y, v.z);
      ss = f0 * ss + f1 * v.w;
    }
    sl = f0 * sl + f1 * v.y;
    mx = up;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) x[e] = f0 * x[e] + f1 * y[e];
  }
  const float inv = sl != 0.f ? 1.f / sl : 0.f;
  const int rr = r + w.tile * a.rows;
  const int64_t head = (((int64_t)w.layer - a.layer0) * a.T + w.off + rr / a.g) * H_q +
                       w.kvh * a.g + rr % a.g;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
    ((__nv_bfloat16 *)a.out)[head * D + lane + 32 * e] = __float2bfloat16_rn(x[e] * inv);
  if (STATS && lane == 0)
    ((float4 *)a.stats)[head] = make_float4(mx * 0.6931471805599453f, sl,
                                            logf(sl) - 0.6931471805599453f * sh * inv, ss * inv);
}

template <int D, int NT, bool STATS>
cudaError_t launch_nt(const Q4AttendArgs &a, int64_t items, cudaStream_t s) {
  using C = Q4Cfg<D, NT>;
  LG_TRY(cudaFuncSetAttribute(q4_attend_kernel<D, NT, STATS>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
  LG_TRY(launch_pdl(q4_attend_kernel<D, NT, STATS>, dim3((unsigned)(items * a.chunks)), kThreads,
                    C::kSmem, s, a));
  return cudaGetLastError();
}

template <int D, bool STATS>
cudaError_t launch_d(const Q4AttendArgs &a, cudaStream_t s) {
  const int64_t items = (int64_t)a.n_layers * a.batch * a.H_kv * a.tiles;
  cudaError_t e = cudaSuccess;
  switch (a.rows) {
    case 8: e = launch_nt<D, 1, STATS>(a, items, s); break;
    case 16: if constexpr (!STATS) e = launch_nt<D, 2, STATS>(a, items, s); break;
    case 24: if constexpr (!STATS) e = launch_nt<D, 3, STATS>(a, items, s); break;
    default: if constexpr (!STATS) e = launch_nt<D, 4, STATS>(a, items, s); break;
  }
  if (e != cudaSuccess) return e;
  if (a.chunks > 1) {
    const int64_t ctas = (items * a.rows + kWarps - 1) / kWarps;
    LG_TRY(launch_pdl(q4_merge_kernel<D, STATS>, dim3((unsigned)ctas), kThreads, 0, s, a));
  }
  return cudaGetLastError();
}

}  // namespace

Q4Grid q4_grid(int n_layers, int batch, int H_kv, int g, int d, int max_new, int max_len, int window,
               int sink) {
  Q4Grid r;
  const int64_t rows = (int64_t)max_new * g;
  r.rows = rows >= 32 ? 32 : (int)((rows + 7) / 8 * 8);
  r.tiles = (int)((rows + r.rows - 1) / r.rows);
  const int64_t items = (int64_t)n_layers * batch * H_kv * r.tiles;
  // key blocks that an item can have: all rows, or the sinks and a window
  int64_t blocks = ((int64_t)max_len + kBn - 1) / kBn;
  if (window)
    blocks = plan_min(blocks, ((int64_t)window + max_new + kBn - 2) / kBn + 1 + ((int64_t)sink + kBn - 1) / kBn);
  // about two waves of the CTAs that the 152 SMs of a GB300 hold, as lengths differ; two blocks at
  // least, as a CTA has its start and end to pay
  const int64_t want = (int64_t)152 * (r.rows <= 16 ? 4 : 2) * 2;
  int64_t per = (blocks * items + want - 1) / want;
  if (per < 2) per = 2;
  if (per > 64) per = 64;
  r.blocks = (int)per;
  r.chunks = (int)((blocks + per - 1) / per);
  // room for any division of as many blocks or fewer, so that a call with a window fits the workspace of
  // one without: a CTA has two blocks and its share of `want` at least, or 64
  const int64_t most = plan_max(plan_min((blocks + 1) / 2, (want + items - 1) / items), (blocks + 63) / 64);
  r.part_bytes = ((size_t)items * most * r.rows * (d + 4) * sizeof(float) + 255) / 256 * 256;
  return r;
}

cudaError_t launch_q4_attend(const Q4AttendArgs &a, int d, cudaStream_t s) {
  if (a.stats) return d == 128 ? launch_d<128, true>(a, s) : launch_d<64, true>(a, s);
  return d == 128 ? launch_d<128, false>(a, s) : launch_d<64, false>(a, s);
}

}  // namespace lg
