// lg_chunk_attend of fp32 caches on the CUDA cores, and the merge of shared items.
//
// chunk_attend_kernel's query tile is BM (64 or 128) rows: the g query heads of BM / g consecutive
// new tokens (row r: token r / g, head r % g), so every key row read serves all of them.  One pass over
// the tile's key blocks with a running maximum m, normaliser l and sum o per row (log2 units):
//   m' = max(m, max s),  p = 2^(s - m'),  l = l 2^(m - m') + sum p,  o = o 2^(m - m') + p V.
// 256 threads as 16 x 16: thread (ty, tx) computes the scores of rows ty TM .. ty TM + TM - 1 and
// keys tx + 16 j, and the results of the same rows and elements 4 tx + 64 j, so that a row's
// probabilities pass between lanes of one half-warp only.
#include <cuda_bf16.h>

#include "lg_chunk_attend.cuh"

namespace lg {
namespace {

constexpr int kThreads = 256;
constexpr int kBn = 64;

__device__ __forceinline__ void load4(const void *p, int64_t i, float *f) {
  const float4 v = *(const float4 *)((const float *)p + i);
  f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
}
__device__ __forceinline__ void store4(void *p, int64_t i, const float *f) {
  *(float4 *)((float *)p + i) = make_float4(f[0], f[1], f[2], f[3]);
}

template <int D, int BM>
struct SimtCfg {
  static constexpr int kRow = D + 4;  // floats of a staged row: 16 rows of 16 bytes, no conflicts
  static constexpr int kSmem =
      (BM * kRow + kBn * kRow + kBn * D + BM * (kBn + 4)) * (int)sizeof(float);
};

template <bool E>
struct Edge {
  static constexpr bool value = E;
};

template <int D, int BM>
__global__ void __launch_bounds__(kThreads) chunk_attend_kernel(ChunkAttendArgs a) {
  constexpr int TM = BM / 16, NC = D / 64, kRow = SimtCfg<D, BM>::kRow, kPRow = kBn + 4;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = sq + BM * kRow, *sv = sk + kBn * kRow, *sp = sv + kBn * D;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int H_q = a.H_kv * a.g;
  pdl_enter();
  ChunkShare sh;
  ChunkWalk<false> w;
  const bool work = chunk_share<false>(a, blockIdx.x, gridDim.x, sh);
  if (work) w.start(a, sh);
  if (tid == 0) put_cut(a, D, gridDim.x, blockIdx.x, work, sh, w);
  for (; work && !w.done(); w.next(a)) {
    if (w.blk0 == w.blk1) continue;
    const int used = w.tokens(a) * a.g;  // rows of the tile that are queries
    const int tok0 = w.off + w.t * a.shape.tok;
    __syncthreads();
    for (int e = tid; e < BM * (D / 4); e += kThreads) {
      const int r = e / (D / 4), c = e % (D / 4) * 4;
      float f[4] = {0.f, 0.f, 0.f, 0.f};
      if (r < used)
        load4(a.q, ((int64_t)(tok0 + r / a.g) * H_q + w.kvh * a.g + r % a.g) * D + c, f);
      *(float4 *)(sq + r * kRow + c) = make_float4(f[0], f[1], f[2], f[3]);
    }
    float o[TM][4 * NC], m[TM], l[TM];
    int qrow[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
      qrow[i] = w.rows.first + (ty * TM + i) / a.g;
#pragma unroll
      for (int k = 0; k < 4 * NC; ++k) o[i][k] = 0.f;
    }
    int open0, open1;
    open_blocks(w.rows, a.shape, w.blocks, open0, open1);
    // rows i0 .. of the keys or values into shared memory, those past the sequence as zeros
    auto copy = [&](float *dst, int row, const void *src, int blk) {
      const int i0 = w.blocks.index(blk) * kBn;
      for (int e = tid; e < kBn * (D / 4); e += kThreads) {
        const int r = e / (D / 4), c = e % (D / 4) * 4;
        const bool in = i0 + r < w.q.n;
        cp_async16_or_zero(dst + r * row + c,
                           (const float *)src + (w.row0 + (in ? i0 + r : 0)) * D + c, in);
      }
      cp_async_commit();
    };
    copy(sk, kRow, a.K, w.blk0);
    for (int blk = w.blk0; blk < w.blk1; ++blk) {
      const int i0 = w.blocks.index(blk) * kBn;
      const bool hides = blk < open0 || blk >= open1;
      copy(sv, D, a.V, blk);  // (on its way while the scores are formed)
      cp_async_wait<1>();
      __syncthreads();
      // scores, even and odd elements summed apart
      float2 acc[TM][4];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        float4 kf[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kf[j] = *(const float4 *)(sk + (tx + 16 * j) * kRow + c);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const float4 qf = *(const float4 *)(sq + (ty * TM + i) * kRow + c);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[i][j] = __ffma2_rn(make_float2(qf.x, qf.y), make_float2(kf[j].x, kf[j].y), acc[i][j]);
            acc[i][j] = __ffma2_rn(make_float2(qf.z, qf.w), make_float2(kf[j].z, kf[j].w), acc[i][j]);
          }
        }
      }
      float alpha[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float s[4], mx = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool sees = !hides || row_sees(w.rows, a.shape, qrow[i], i0 + tx + 16 * j);
          s[j] = sees ? (acc[i][j].x + acc[i][j].y) * a.qscale : -INFINITY;
          mx = fmaxf(mx, s[j]);
        }
#pragma unroll
        for (int off = 8; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float base = mx == -INFINITY ? 0.f : mx;
        alpha[i] = exp2_fast(m[i] - base);
        m[i] = mx;
        l[i] *= alpha[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = exp2_fast(s[j] - base);
          l[i] += p;
          sp[(ty * TM + i) * kPRow + tx + 16 * j] = p;
        }
      }
      __syncthreads();  // the keys have been read (and a half-warp's probabilities are written)
      if (blk + 1 < w.blk1)
        copy(sk, kRow, a.K, blk + 1);
      else
        cp_async_commit();
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int k = 0; k < 4 * NC; ++k) o[i][k] *= alpha[i];
      cp_async_wait<1>();
      __syncthreads();
      auto sums = [&](auto edge) {
#pragma unroll 2
        for (int r = 0; r < kBn; r += 4) {
          float4 p[TM];
#pragma unroll
          for (int i = 0; i < TM; ++i) p[i] = *(const float4 *)(sp + (ty * TM + i) * kPRow + r);
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int k = 0; k < NC; ++k) {
              const float4 v = *(const float4 *)(sv + (r + rr) * D + 4 * tx + 64 * k);
#pragma unroll
              for (int i = 0; i < TM; ++i) {
                const float pr = rr == 0 ? p[i].x : rr == 1 ? p[i].y : rr == 2 ? p[i].z : p[i].w;
                // a hidden row has probability 0 and may hold anything
                const bool add = !decltype(edge)::value || pr != 0.f;
                float2 *oo = (float2 *)&o[i][4 * k];
                const float2 pp = make_float2(pr, pr);
                oo[0] = __ffma2_rn(pp, add ? make_float2(v.x, v.y) : make_float2(0.f, 0.f), oo[0]);
                oo[1] = __ffma2_rn(pp, add ? make_float2(v.z, v.w) : make_float2(0.f, 0.f), oo[1]);
              }
            }
        }
      };
      if (hides)
        sums(Edge<true>{});
      else
        sums(Edge<false>{});
      __syncthreads();  // the values have been read
    }
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int r = ty * TM + i;
#pragma unroll
      for (int off = 8; off; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
      if (r >= used) continue;
      if (w.whole()) {
        const float inv = l[i] != 0.f ? 1.f / l[i] : 0.f;
        const int64_t dst = ((int64_t)(tok0 + r / a.g) * H_q + w.kvh * a.g + r % a.g) * D;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = o[i][4 * k + e] * inv;
          store4(a.out, dst + 4 * tx + 64 * k, f);
        }
      } else {
#pragma unroll
        for (int k = 0; k < NC; ++k)
          *part_at(a, D, blockIdx.x, w.slot(), tx + 16 * k, r) =
              make_float4(o[i][4 * k], o[i][4 * k + 1], o[i][4 * k + 2], o[i][4 * k + 3]);
        if (tx == 0) *part_ml(a, D, gridDim.x, blockIdx.x, w.slot(), r) = make_float2(m[i], l[i]);
      }
    }
  }
}

// The same for at most 16 query rows of a kv-head, where reading the cache is all of the work: a warp
// takes eight keys of every block, a row of them at a load (two of 64 elements), each lane four
// elements.  The products of a key with all R query rows are summed over the lanes by halving (each
// level hands half of the rows over), which leaves a row's score to 32 / R lanes; its weights go
// through shared memory to all lanes, which add weight x value to R x 4 sums of their own.  m lags
// as in the tensor-core kernels.  The eight warps' results are merged at the end of a piece.
template <int D, int R>
struct FewF32 {
  static constexpr int kLanes = D / 4;          // lanes of a row
  static constexpr int kKeys = 32 / kLanes;     // keys of a load
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kSmem =
      kWarps * R * (D + 2) * (int)sizeof(float);  // results, maxima and normalisers
};
constexpr int kFewKeys = kBn / (kThreads / 32);  // of a warp in a block
constexpr float kLazy = 8.f;

template <int D, int R>
__global__ void __launch_bounds__(kThreads, R == 4 ? 2 : 1)
    chunk_attend_few_f32_kernel(ChunkAttendArgs a) {
  using C = FewF32<D, R>;
  constexpr int LPR = C::kLanes, KPL = C::kKeys, NL = kFewKeys / KPL;  // loads of a block
  extern __shared__ __align__(16) float smem[];
  __shared__ __align__(16) float s_p[C::kWarps][kFewKeys + 1][R];  // weights; what sums are scaled by
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int half = lane / LPR, el = lane % LPR;       // key of a load, group of four elements
  const int row = el / (LPR / R);                     // the row whose scores this lane keeps
  const bool keeper = el % (LPR / R) == 0;
  const int H_q = a.H_kv * a.g;
  float *s_o = smem, *s_m = smem + C::kWarps * R * D, *s_l = s_m + C::kWarps * R;
  pdl_enter();
  ChunkShare sh;
  ChunkWalk<true> w;
  const bool work = chunk_share<true>(a, blockIdx.x, gridDim.x, sh);
  if (work) w.start(a, sh);
  if (tid == 0) put_cut(a, D, gridDim.x, blockIdx.x, work, sh, w);
  for (; work && !w.done(); w.next(a)) {
    if (w.blk0 == w.blk1) continue;
    const int used = w.tokens(a) * a.g, tok0 = w.off + w.t * a.shape.tok;
    const int qrow = w.rows.first + row / a.g;
    float4 q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      q[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < used)
        q[r] = *(const float4 *)((const float *)a.q +
                                 ((int64_t)(tok0 + r / a.g) * H_q + w.kvh * a.g + r % a.g) * D +
                                 4 * el);
    }
    float2 o[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) o[r][0] = o[r][1] = make_float2(0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    int open0, open1;
    open_blocks(w.rows, a.shape, w.blocks, open0, open1);
    for (int blk = w.blk0; blk < w.blk1; ++blk) {
      const int i0 = w.blocks.index(blk) * kBn + warp * kFewKeys + half;  // this lane's first key
      const bool hides = blk < open0 || blk >= open1;
      float4 k[NL], v[NL];
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const int i = i0 + j * KPL;
        k[j] = v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < w.q.n) {
          k[j] = *(const float4 *)((const float *)a.K + (w.row0 + i) * D + 4 * el);
          v[j] = *(const float4 *)((const float *)a.V + (w.row0 + i) * D + 4 * el);
        }
      }
      float sc[NL], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        float x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float2 t = __fmul2_rn(make_float2(q[r].x, q[r].y), make_float2(k[j].x, k[j].y));
          t = __ffma2_rn(make_float2(q[r].z, q[r].w), make_float2(k[j].z, k[j].w), t);
          x[r] = t.x + t.y;
        }
        HeadReduce<R, LPR / 2>::run(x, lane);
        const int i = i0 + j * KPL;
        const bool sees = !hides || row_sees(w.rows, a.shape, qrow, i);
        sc[j] = sees ? x[0] * a.qscale : -INFINITY;
        top = fmaxf(top, sc[j]);
      }
      if (KPL == 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
      const bool rise = top > m + kLazy || (m == -INFINITY && top > m);
      if (__any_sync(0xffffffffu, rise)) {
        const float m1 = rise ? top : m;
        const float f = rise ? exp2_fast(m - m1) : 1.f;
        m = m1;
        l *= f;
        __syncwarp();
        if (keeper && half == 0) s_p[warp][kFewKeys][row] = f;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float fr = s_p[warp][kFewKeys][r];
          o[r][0] = __fmul2_rn(o[r][0], make_float2(fr, fr));
          o[r][1] = __fmul2_rn(o[r][1], make_float2(fr, fr));
        }
      }
      const float base = m == -INFINITY ? 0.f : m;
      __syncwarp();
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const float p = exp2_fast(sc[j] - base);
        l += p;
        if (keeper) s_p[warp][j * KPL + half][row] = p;
      }
      __syncwarp();
      auto sums = [&](auto edge) {
#pragma unroll
        for (int j = 0; j < NL; ++j)
#pragma unroll
          for (int r = 0; r < R; r += 4) {
            const float4 p4 = *(const float4 *)&s_p[warp][j * KPL + half][r];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = e == 0 ? p4.x : e == 1 ? p4.y : e == 2 ? p4.z : p4.w;
              // a hidden row has weight 0 and may hold anything
              const bool add = !decltype(edge)::value || p != 0.f;
              o[r + e][0] = __ffma2_rn(make_float2(p, p),
                                       add ? make_float2(v[j].x, v[j].y) : make_float2(0.f, 0.f),
                                       o[r + e][0]);
              o[r + e][1] = __ffma2_rn(make_float2(p, p),
                                       add ? make_float2(v[j].z, v[j].w) : make_float2(0.f, 0.f),
                                       o[r + e][1]);
            }
          }
      };
      if (hides)
        sums(Edge<true>{});
      else
        sums(Edge<false>{});
    }
    // the warps' results meet in shared memory
    if (KPL == 2) {
      l += __shfl_xor_sync(0xffffffffu, l, 16);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[r][e].x += __shfl_xor_sync(0xffffffffu, o[r][e].x, 16);
          o[r][e].y += __shfl_xor_sync(0xffffffffu, o[r][e].y, 16);
        }
    }
    __syncthreads();  // (the previous piece's have been read)
    if (half == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        *(float4 *)(s_o + (warp * R + r) * D + 4 * el) =
            make_float4(o[r][0].x, o[r][0].y, o[r][1].x, o[r][1].y);
      if (keeper) {
        s_m[warp * R + row] = m;
        s_l[warp * R + row] = l;
      }
    }
    __syncthreads();
    for (int e = tid; e < used * LPR; e += kThreads) {
      const int r = e / LPR, c = e % LPR;
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int x = 0; x < C::kWarps; ++x) mx = fmaxf(mx, s_m[x * R + r]);
      const float base = mx == -INFINITY ? 0.f : mx;
      float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int x = 0; x < C::kWarps; ++x) {
        const float f = exp2_fast(s_m[x * R + r] - base);
        const float4 y = *(const float4 *)(s_o + (x * R + r) * D + 4 * c);
        sum += s_l[x * R + r] * f;
        t.x += y.x * f, t.y += y.y * f, t.z += y.z * f, t.w += y.w * f;
      }
      if (w.whole()) {
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        const float f[4] = {t.x * inv, t.y * inv, t.z * inv, t.w * inv};
        store4(a.out, ((int64_t)(tok0 + r / a.g) * H_q + w.kvh * a.g + r % a.g) * D + 4 * c, f);
      } else {
        *part_at(a, D, blockIdx.x, w.slot(), c, r) = t;
        if (c == 0) *part_ml(a, D, gridDim.x, blockIdx.x, w.slot(), r) = make_float2(mx, sum);
      }
    }
  }
}

// Merge of the item that CTA c's start is the first to cut, c = blockIdx.x + 1, from the parts of
// CTAs c - 1, c, ...: 32 rows a CTA, a lane each, the elements spread over the eight warps; the rows
// leave through shared memory, 16 bytes a thread.  SHARE, for items of few rows and many parts: two or
// four lanes share a row and take every second or fourth part (a token over 16000 rows, bf16, two
// kv-heads of 64, 76 parts: 24.9 us without, 14.4; eight of 128, 19 parts: 17.8 and 14.9; eight
// sequences of them, three parts: 48.0 without, 49.3; one over 200 rows: 9.3 and 9.9).  The loads of
// kAtOnce parts wait together: 8 where items are short and have many, 4 where they are long (fewer
// registers, more CTAs an SM; 12 took 16 x 7 proposed tokens from 23.0 to 25.5 us).
constexpr int kMergeRows = 32;

template <typename T, int D, int kAtOnce, bool SHARE>
__global__ void __launch_bounds__(kThreads) chunk_merge_kernel(ChunkAttendArgs a, int G) {
  constexpr int NE = D / 4 / (kThreads / 32);  // groups of four elements a thread
  constexpr int kRow = D * (int)sizeof(T) + 16;
  __shared__ __align__(16) uint8_t s_out[kMergeRows * kRow];
  const int c = blockIdx.x + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_enter();
  const ChunkCut w = *cut_at(a, D, G, c);
  if (cta_status_bad(a.status)) return;
  const int r0 = blockIdx.y * kMergeRows;
  if (w.parts == 0 || r0 >= w.used) return;
  // log2 of the lanes of a row
  const int share = !SHARE || w.parts <= kAtOnce ? 0
                    : w.used <= 8 && w.parts > 2 * kAtOnce ? 2 : w.used <= 16 ? 1 : 0;
  const int r = r0 + (lane & (kMergeRows >> share) - 1), first = lane / (kMergeRows >> share);
  float m = -INFINITY, l = 0.f;
  float4 o[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  int before = 0;
  for (int p0 = 0; p0 < w.parts; p0 += kAtOnce << share) {
    float2 ml[kAtOnce];
    float4 x[kAtOnce][NE];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int p = p0 + (k << share) + first;
      ml[k] = make_float2(-INFINITY, 0.f);
      const int64_t y = w.in + p * w.step;
      if (share && p > 0) before = cut_block(y - w.step, w.cost, w.blocks, a.shape.bn2);
      const int from = before, to = cut_block(y, w.cost, w.blocks, a.shape.bn2);
      before = to;
      // one part has every block and wrote the result
      const bool whole = p < w.parts && from == 0 && to == w.blocks;
      if (SHARE ? __any_sync(0xffffffffu, whole) : whole) return;
      if (p >= w.parts || from == to || r >= w.used) continue;
      const int cta = c - 1 + p, slot = p == 0 ? 1 : 0;
      ml[k] = *part_ml(a, D, G, cta, slot, r);
#pragma unroll
      for (int e = 0; e < NE; ++e) x[k][e] = *part_at(a, D, cta, slot, warp * NE + e, r);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (ml[k].x == -INFINITY && ml[k].y == 0.f) continue;  // (no part, or nothing was seen in it)
      const float mx = fmaxf(m, ml[k].x), base = mx == -INFINITY ? 0.f : mx;
      const float f0 = exp2_fast(m - base), f1 = exp2_fast(ml[k].x - base);
      m = mx;
      l = l * f0 + ml[k].y * f1;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        o[e].x = o[e].x * f0 + x[k][e].x * f1;
        o[e].y = o[e].y * f0 + x[k][e].y * f1;
        o[e].z = o[e].z * f0 + x[k][e].z * f1;
        o[e].w = o[e].w * f0 + x[k][e].w * f1;
      }
    }
  }
  for (int off = kMergeRows >> share; off < kMergeRows; off <<= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, m, off), l1 = __shfl_xor_sync(0xffffffffu, l, off);
    const float mx = fmaxf(m, m1), base = mx == -INFINITY ? 0.f : mx;
    const float f0 = exp2_fast(m - base), f1 = exp2_fast(m1 - base);
    m = mx;
    l = l * f0 + l1 * f1;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      o[e].x = o[e].x * f0 + __shfl_xor_sync(0xffffffffu, o[e].x, off) * f1;
      o[e].y = o[e].y * f0 + __shfl_xor_sync(0xffffffffu, o[e].y, off) * f1;
      o[e].z = o[e].z * f0 + __shfl_xor_sync(0xffffffffu, o[e].z, off) * f1;
      o[e].w = o[e].w * f0 + __shfl_xor_sync(0xffffffffu, o[e].w, off) * f1;
    }
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    if (first) break;
    uint8_t *at = s_out + (r - r0) * kRow + (warp * NE + e) * 4 * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
      *(float4 *)at = make_float4(o[e].x * inv, o[e].y * inv, o[e].z * inv, o[e].w * inv);
    } else {
      const __nv_bfloat162 h[2] = {__floats2bfloat162_rn(o[e].x * inv, o[e].y * inv),
                                   __floats2bfloat162_rn(o[e].z * inv, o[e].w * inv)};
      *(uint2 *)at = *(const uint2 *)h;
    }
  }
  __syncthreads();
  constexpr int kPer = D * (int)sizeof(T) / 16;  // 16-byte pieces of a row
  for (int i = threadIdx.x; i < kMergeRows * kPer; i += kThreads) {
    const int rr = i / kPer, q = r0 + rr;
    if (q >= w.used) break;
    const int64_t dst = ((int64_t)(w.tok0 + q / a.g) * (a.H_kv * a.g) + w.kvh * a.g + q % a.g) * D;
    *(uint4 *)((T *)a.out + dst + i % kPer * (16 / (int)sizeof(T))) =
        *(const uint4 *)(s_out + rr * kRow + i % kPer * 16);
  }
}

cudaError_t launch_f32(void (*kern)(ChunkAttendArgs), int smem, const ChunkAttendArgs &a, int G,
                       cudaStream_t s) {
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  LG_TRY(launch_pdl(kern, G, kThreads, smem, s, a));
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_merge_typed(const ChunkAttendArgs &a, int G, cudaStream_t s) {
  const dim3 grid(G - 1, (a.rows + kMergeRows - 1) / kMergeRows);
  // more than eight parts an item, and blocks for them
  if (a.rows <= 16 && (int64_t)a.batch * a.H_kv * 8 < G && a.max_len > 8 << a.shape.bn2)
    LG_TRY(launch_pdl(chunk_merge_kernel<T, D, 8, true>, grid, kThreads, 0, s, a, G));
  else if (a.rows <= 64)
    LG_TRY(launch_pdl(chunk_merge_kernel<T, D, 8, false>, grid, kThreads, 0, s, a, G));
  else
    LG_TRY(launch_pdl(chunk_merge_kernel<T, D, 4, false>, grid, kThreads, 0, s, a, G));
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(ChunkAttendArgs &a, int G, cudaStream_t s) {
  switch (a.rows) {
    case 4: return launch_f32(chunk_attend_few_f32_kernel<D, 4>, FewF32<D, 4>::kSmem, a, G, s);
    case 8: return launch_f32(chunk_attend_few_f32_kernel<D, 8>, FewF32<D, 8>::kSmem, a, G, s);
    case 16: return launch_f32(chunk_attend_few_f32_kernel<D, 16>, FewF32<D, 16>::kSmem, a, G, s);
  }
  if (a.rows == 64)
    return launch_f32(chunk_attend_kernel<D, 64>, SimtCfg<D, 64>::kSmem, a, G, s);
  return launch_f32(chunk_attend_kernel<D, 128>, SimtCfg<D, 128>::kSmem, a, G, s);
}

}  // namespace

cudaError_t launch_chunk_merge(const ChunkAttendArgs &a, int dtype, int d, int G, cudaStream_t s) {
  if (dtype == LG_BF16)
    return d == 128 ? launch_merge_typed<__nv_bfloat16, 128>(a, G, s)
                    : launch_merge_typed<__nv_bfloat16, 64>(a, G, s);
  return d == 128 ? launch_merge_typed<float, 128>(a, G, s)
                  : launch_merge_typed<float, 64>(a, G, s);
}

ChunkGrid chunk_grid(int dtype, int d, int g, int max_new) {
  if (dtype == LG_BF16) return chunk_grid_tc(d, g, max_new);
  ChunkGrid r;
  const int64_t rows = (int64_t)max_new * g;
  r.rows = rows <= 4 ? 4 : rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 64 ? 64 : 128;
  // what the 152 SMs of a GB300 hold at once (on fewer the others follow: no CTA waits for another)
  r.ctas = 152 * (r.rows == 4 ? 2 : 1);
  r.tok = r.rows / g;
  r.bn2 = 6;
  return r;
}

cudaError_t launch_chunk_attend(ChunkAttendArgs &a, int dtype, int d, int G, cudaStream_t s) {
  cudaError_t e;
  if (dtype == LG_BF16)
    e = launch_chunk_attend_tc(a, d, G, s);
  else
    e = d == 128 ? launch_d<128>(a, G, s) : launch_d<64>(a, G, s);
  if (e != cudaSuccess) return e;
  return launch_chunk_merge(a, dtype, d, G, s);
}

}  // namespace lg
