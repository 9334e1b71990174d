// lg_chunk_attend of bf16 caches for few query rows of a kv-head (a token, or some proposed tokens,
// a sequence): the call reads the cache once and computes little, so the products are turned round,
//   S^T = K Q^T  (M = 128 keys, N query rows),  O^T += V^T P^T  (M = head elements),
// and no part of them is padding.  A thread holds one key's scores of 16 or 32 of the N rows (N = 16,
// 32 or 64: row r is token r / g, head r % g; one group of four warps takes 16 rows, two take 32 or
// 64); it exponentiates them, adds them to its own sums of the normalisers and writes them to its
// key's row of P^T in shared memory, the products' second operand.  The maxima are the group's: as in
// the kernel for many rows they may lag by a factor 2^8, so a block asks only whether any score passed
// that bound (one barrier), and the exact maxima are formed in the first block, when one did, and when
// a query that has seen nothing so far sees a row (a window may begin in a later block for a tile's
// later tokens; until then the query has no maximum that its weights could be measured by).
//
// Scores are two blocks ahead of the sums (two buffers of S^T and P^T), and the ring holds five
// blocks of keys or values.
//
// Warps: the keys' (and the results': a thread a head element), one that walks along the work and
// copies, one that issues the products, two that clear what is not a number from values of blocks
// that hide a row from a query.
#include <stddef.h>

#include "lg_chunk_tc.cuh"

namespace lg {
namespace {

constexpr int kBn = 128;            // rows of a key block
constexpr int kPBytes = kBn * 128;  // a buffer of P^T: 128-byte rows, swizzled
constexpr float kLazy = 8.f;
constexpr float kNothing = -3e38f;  // below every score by more than kLazy, and finite
constexpr uint32_t kTmemCols = 256;

template <int D, int N>
struct FewCfg {
  static constexpr int kBoxes = D / 64;
  static constexpr int kTile = kBn * D * 2;
  static constexpr int kQBox = N * 128;
  static constexpr int kQBytes = (kBoxes * kQBox + 1023) / 1024 * 1024;
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr int kGroups = N > 16 ? 2 : 1;  // groups of four warps that share a block's keys
  static constexpr int kCols = N / kGroups;       // query rows of a thread
  static constexpr int kWarps = 4 * kGroups;      // ... and the other roles' first warp
  static constexpr int kThreads = 32 * (kWarps + 4);
  static constexpr int kSmem = kQBytes + 2 * kPBytes + kStages * kTile + 1024;
};

template <int ST, int N>
struct FewBars {
  uint64_t full[ST], empty[ST], fixed[ST];
  uint64_t q_full, q_empty;
  uint64_t s_full[2], p_full[2];
  uint64_t o_full[2], o_free;  // sums of even and odd blocks ready: a wait is never two phases away
  TcQueue queue;
  uint32_t tmem;
  volatile int give_up;
  __align__(16) float col[4][N];  // a warp's maxima or normalisers
  // the maxima in use; what the sums so far are multiplied by (both read as 16-byte vectors)
  __align__(16) float m[N];
  __align__(16) float f[N];
};

// a barrier of a group's 128 key threads; with a condition: whether it held for any
__device__ __forceinline__ void keys_sync(int group) {
  asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory");
}
__device__ __forceinline__ bool keys_any(int group, bool p) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, 128, p;\n"
      " selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)p), "r"(group + 1)
      : "memory");
  return r != 0;
}

template <int N>
__device__ __forceinline__ void load_cols(uint32_t addr, uint32_t *v) {
  if constexpr (N == 16) {
    tmem_load16(addr, v);
  } else {
#pragma unroll
    for (int x = 0; x < N; x += 32) tmem_load32(addr + x, v + x);
  }
  tmem_wait_load();
}

template <int N>
__device__ __forceinline__ void store_cols(uint32_t addr, const uint32_t *v) {
  if constexpr (N == 16) {
    tmem_store16(addr, v);
  } else {
#pragma unroll
    for (int x = 0; x < N; x += 32) tmem_store32(addr + x, v + x);
  }
  tmem_wait_store();
}

// bit q: query row q (token q / g of the tile) sees row i
__device__ __forceinline__ uint64_t columns_seeing(const TileRows &r, const ChunkShape &s, int g,
                                                   int i) {
  auto below = [](int64_t n) {  // bits 0 .. n - 1
    return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
  };
  const uint64_t from = ~below(((int64_t)i - r.first) * g);  // tokens at row i or behind it
  if (s.window == 0 || i < s.sink) return from;
  return from & below(((int64_t)i + s.window - r.first) * g);
}

template <int D, int N>
__global__ void __launch_bounds__((FewCfg<D, N>::kThreads), 1)
    chunk_attend_few_kernel(const __grid_constant__ CUtensorMap mq,
                            const __grid_constant__ CUtensorMap mk,
                            const __grid_constant__ CUtensorMap mv, ChunkAttendArgs a) {
  using C = FewCfg<D, N>;
  using B = FewBars<C::kStages, N>;
  static_assert(offsetof(B, m) % 16 == 0 && offsetof(B, f) % 16 == 0 && alignof(B) % 16 == 0,
                "read as 16-byte vectors");
  constexpr int ST = C::kStages, NC = C::kCols, W0 = C::kWarps;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) FewBars<ST, N> bars;
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sq = smem, *sp = sq + C::kQBytes, *ring = sp + 2 * kPBytes;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 3);
      mbar_init(&bars.fixed[i], 2);
    }
    mbar_init(&bars.q_full, 1);
    mbar_init(&bars.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], W0);
      mbar_init(&bars.o_full[i], 1);
    }
    mbar_init(&bars.o_free, W0);
    bars.queue.init(3 + W0);  // the products, two clearing warps, the keys' warps
    bars.give_up = 0;
    mbar_fence_init();
  }
  if (warp == W0 + 1) tmem_alloc(&bars.tmem, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_enter();
  const uint32_t tmem = bars.tmem;  // S^T at columns 0 and N, O^T at 2 N

  if (warp == W0) {
    ChunkShare sh;
    const bool work = chunk_share<true>(a, blockIdx.x, gridDim.x, sh);
    if (lane == 0) {
      ChunkWalk<true> w;
      uint32_t n = 0, pieces = 0;
      bool ok = true;
      auto load = [&](const CUtensorMap *map, int row) {
        const uint32_t st = n % ST;
        ok = ok && tc_wait(bars, &bars.empty[st], ((n / ST) & 1) ^ 1);
        if (!ok) return;
        mbar_arrive_expect_tx(&bars.full[st], C::kTile);
#pragma unroll
        for (int x = 0; x < C::kBoxes; ++x)
          tma_box_2d(ring + st * C::kTile + x * (kBn * 128), map, 64 * x, row, &bars.full[st]);
        ++n;
      };
      if (work) w.start(a, sh);
      const ChunkWalk<true> first = w;
      for (; work && ok && !w.done(); w.next(a)) {
        if (w.blk0 == w.blk1) continue;
        const int r0 = (int)w.row0;
        ok = tc_wait(bars, &bars.q_empty, (pieces & 1) ^ 1);
        if (!ok) break;
        mbar_arrive_expect_tx(&bars.q_full, C::kBoxes * a.shape.tok * a.g * 128);
#pragma unroll
        for (int x = 0; x < C::kBoxes; ++x)
          tma_box_3d(sq + x * C::kQBox, &mq, 64 * x, w.kvh * a.g, w.off + w.t * a.shape.tok,
                     &bars.q_full);
        // keys a block ahead of the values, as the products take them
        load(&mk, r0 + w.blocks.index(w.blk0) * kBn);
        ok = ok && bars.queue.put(bars, pieces, w, a);
        ++pieces;
        for (int j = w.blk0; ok && j < w.blk1; ++j) {
          if (j + 1 < w.blk1) load(&mk, r0 + w.blocks.index(j + 1) * kBn);
          load(&mv, r0 + w.blocks.index(j) * kBn);
        }
      }
      if (ok) bars.queue.end(bars, pieces);
      put_cut(a, D, gridDim.x, blockIdx.x, work, sh, first);
    }
  } else if (warp == W0 + 1) {
    const bool one = elect_one();
    uint32_t n = 0, c = 0;
    bool ok = true;
    constexpr uint32_t kIdS = mma_idesc(128, N, false, false);
    constexpr uint32_t kIdO = mma_idesc(128, N, true, true);
    // a head of 64 elements fills 64 of the 128 rows: the others repeat them
    constexpr uint32_t kLboV = D == 128 ? kBn * 128 : 0;
    const uint32_t q_lo = desc_lo(smem_addr(sq), 16), p_lo = desc_lo(smem_addr(sp), 16);
    const uint32_t k_lo = desc_lo(smem_addr(ring), 16), v_lo = desc_lo(smem_addr(ring), kLboV);
    auto wait_full = [&](uint32_t i) {
      ok = ok && tc_wait_warp(bars, &bars.full[i % ST], (i / ST) & 1);
    };
    for (uint32_t pc = 0;; ++pc) {
      ok = bars.queue.wait(bars, pc);
      if (!ok) break;
      const TcPiece &p = bars.queue.at(pc);
      const int blk0 = uniform(p.blk0), blocks = uniform(p.blk1) - blk0;
      if (uniform(p.blk1) < 0) break;
      const int open0 = uniform(p.open0) - blk0, open1 = uniform(p.open1) - blk0;
      __syncwarp();
      if (one) bars.queue.done(pc);
      ok = tc_wait_warp(bars, &bars.q_full, pc & 1);
      auto k_at = [&](int j) { return n + (j == 0 ? 0 : 2 * j - 1); };
      auto scores = [&](int j) {
        wait_full(k_at(j));
        if (!ok) return;
        tc_fence_after();
        const uint32_t b = (c + j) & 1, k0 = k_lo + k_at(j) % ST * (C::kTile >> 4);
        if (one) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            tc_mma_ss(tmem + b * N, k0 + (((k / 4) * (kBn * 128) + (k % 4) * 32) >> 4),
                      q_lo + (((k / 4) * C::kQBox + (k % 4) * 32) >> 4), kIdS, k > 0);
          tc_commit(&bars.s_full[b]);
          tc_commit(&bars.empty[k_at(j) % ST]);
          if (j + 1 == blocks) tc_commit(&bars.q_empty);
        }
      };
      scores(0);
      for (int j = 0; ok && j < blocks; ++j) {
        if (j + 1 < blocks) scores(j + 1);
        const uint32_t iv = n + (j + 1 < blocks ? 2 * j + 2 : 2 * j + 1), b = (c + j) & 1;
        // (the copy before the clearing: its arrival says that the ring's slot has been through the
        // clearing warps before, and so which phase of `fixed` the parity means)
        wait_full(iv);
        if (j < open0 || j >= open1)
          ok = ok && tc_wait_warp(bars, &bars.fixed[iv % ST], (iv / ST) & 1);
        if (j == 0) ok = ok && tc_wait_warp(bars, &bars.o_free, (pc & 1) ^ 1);
        ok = ok && tc_wait_warp(bars, &bars.p_full[b], ((c + j) >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        const uint32_t v0 = v_lo + iv % ST * (C::kTile >> 4), p0 = p_lo + b * (kPBytes >> 4);
        if (one) {
#pragma unroll
          for (int k = 0; k < kBn / 16; ++k)
            tc_mma_ss(tmem + 2 * N, v0 + (k * 2048 >> 4), p0 + (k * 2048 >> 4), kIdO,
                      j > 0 || k > 0);
          tc_commit(&bars.o_full[b]);
          tc_commit(&bars.empty[iv % ST]);
        }
      }
      if (!ok) break;
      c += blocks;
      n += 2 * blocks;
    }
  } else if (warp >= W0 + 2) {
    uint32_t n = 0;
    bool ok = true;
    for (uint32_t pc = 0; ok; ++pc) {
      ok = bars.queue.wait(bars, pc);
      if (!ok) break;
      TcPiece &p = bars.queue.at(pc);
      if (p.blk1 < 0) break;
      const int blocks = p.blk1 - p.blk0;
      for (int i = 0; i < 2 * blocks; ++i, ++n) {
        // the i-th copy of the piece: the values of block j, or keys
        const int j = i == 2 * blocks - 1 ? blocks - 1 : i >= 2 && !(i & 1) ? i / 2 - 1 : -1;
        ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.full[n % ST], (n / ST) & 1));
        if (!ok) break;
        if (j >= 0 && p.hides(p.blk0 + j)) {
          const int i0 = p.blocks.index(p.blk0 + j) * kBn;
          if (clear_block<C::kTile, kBn>(ring + n % ST * C::kTile, i0, p.n, tid - 32 * (W0 + 2), 64))
            p.bad = 1;
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (lane == 0) {
          mbar_arrive(&bars.fixed[n % ST]);
          mbar_arrive(&bars.empty[n % ST]);
        }
      }
      __syncwarp();
      if (lane == 0) bars.queue.done(pc);
    }
  } else {
    const int grp = warp >> 2, q0 = grp * NC;  // this thread's query rows: q0 .. q0 + NC - 1
    const int key = tid & 127;                 // of a block; of the results: the head element
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    uint32_t c = 0;
    bool ok = true;
    for (uint32_t pc = 0; ok; ++pc) {
      ok = bars.queue.wait(bars, pc);
      if (keys_any(grp, !ok)) break;
      const TcPiece &w = bars.queue.at(pc);
      if (w.blk1 < 0) break;
      const int used = w.tokens * a.g;
      // base: the maxima in use (kNothing while a query has seen nothing: its first score passes the
      // bound, and its hidden rows' weights are 0), l: normalisers in pairs
      float base[NC];
      float2 l2[NC / 2];
#pragma unroll
      for (int q = 0; q < NC; ++q) base[q] = 0.f;
#pragma unroll
      for (int q = 0; q < NC / 2; ++q) l2[q] = make_float2(0.f, 0.f);
      // (rows of the tile that are no query, which may hold anything: their scores are always below
      // it, so that they never ask for new maxima, which would round the queries' weights otherwise)
      if (key < NC) bars.m[q0 + key] = q0 + key < used ? -INFINITY : INFINITY;
      const float2 sc = make_float2(a.qscale, a.qscale);
      for (int blk = w.blk0; blk < w.blk1; ++blk, ++c) {
        const uint32_t b = c & 1;
        const int i0 = w.blocks.index(blk) * kBn;
        const bool hides = w.hides(blk);
        const uint64_t see = hides ? columns_seeing(w.rows, a.shape, a.g, i0 + key) >> q0 : ~0ull;
        ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.s_full[b], (c >> 1) & 1));
        // a role that gave up is seen by every key warp before the barriers below
        if (keys_any(grp, !ok)) {
          ok = false;
          break;
        }
        tc_fence_after();
        uint32_t u[NC];
        load_cols<NC>(tmem + b * N + q0 + lanes, u);
        float *v = (float *)u;
        if (hides) {
#pragma unroll
          for (int q = 0; q < NC; ++q)
            if (!(see >> q & 1)) v[q] = -INFINITY;
        }
        float2 z[NC / 2];  // scores over the maxima in use
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < NC; q += 2) {
          z[q / 2] = __ffma2_rn(make_float2(v[q], v[q + 1]), sc, make_float2(-base[q], -base[q + 1]));
          top = max3(top, z[q / 2].x, z[q / 2].y);
        }
        if (keys_any(grp, top > kLazy || blk == w.blk0)) {
          float mine = -INFINITY;  // lane q: the warp's maximum of row q
#pragma unroll
          for (int q = 0; q < NC; ++q) {
            const float x = warp_max(v[q]);
            if (lane == q) mine = x;
          }
          if (lane < NC) bars.col[warp & 3][q0 + lane] = mine;
          keys_sync(grp);
          if (key < NC) {
            const int q = q0 + key;
            const float x = fmaxf(fmaxf(bars.col[0][q], bars.col[1][q]),
                                  fmaxf(bars.col[2][q], bars.col[3][q])) * a.qscale;
            const float m0 = bars.m[q], m1 = fmaxf(m0, x);
            bars.m[q] = m1;
            bars.f[q] = m1 == -INFINITY ? 0.f : exp2_fast(m0 - m1);
          }
          keys_sync(grp);
          float f[NC];
#pragma unroll
          for (int q = 0; q < NC; q += 4) {
            const float4 m4 = *(const float4 *)&bars.m[q0 + q], f4 = *(const float4 *)&bars.f[q0 + q];
            base[q] = m4.x, base[q + 1] = m4.y, base[q + 2] = m4.z, base[q + 3] = m4.w;
            f[q] = f4.x, f[q + 1] = f4.y, f[q + 2] = f4.z, f[q + 3] = f4.w;
          }
#pragma unroll
          for (int q = 0; q < NC; ++q)
            if (base[q] == -INFINITY) base[q] = kNothing;
#pragma unroll
          for (int q = 0; q < NC; q += 2) {
            z[q / 2] = __ffma2_rn(make_float2(v[q], v[q + 1]), sc, make_float2(-base[q], -base[q + 1]));
            l2[q / 2].x *= f[q];
            l2[q / 2].y *= f[q + 1];
          }
          if (blk > w.blk0) {
            ok = __all_sync(0xffffffffu,
                            tc_wait(bars, &bars.o_full[(c - 1) & 1], ((c - 1) >> 1) & 1));
            if (keys_any(grp, !ok)) {
              ok = false;
              break;
            }
            tc_fence_after();
            uint32_t o[NC];
            load_cols<NC>(tmem + 2 * N + q0 + lanes, o);
#pragma unroll
            for (int q = 0; q < NC; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * f[q]);
            store_cols<NC>(tmem + 2 * N + q0 + lanes, o);
            tc_fence_before();
          }
        }
        uint8_t *row = sp + b * kPBytes + key * 128;
#pragma unroll
        for (int q = 0; q < NC; q += 8) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float2 p = z[q / 2 + e];
            p.x = exp2_fast(p.x);
            p.y = exp2_fast(p.y);
            l2[q / 2 + e] = __fadd2_rn(l2[q / 2 + e], p);
            const __nv_bfloat162 y = __floats2bfloat162_rn(p.x, p.y);
            h[e] = *(const uint32_t *)&y;
          }
          *(uint4 *)(row + ((((q0 + q) / 8) ^ (key & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full[b]);
      }
      if (!ok) break;
      // normalisers: a warp's sums, then the CTA's
      float l[NC];
#pragma unroll
      for (int q = 0; q < NC / 2; ++q) l[2 * q] = l2[q].x, l[2 * q + 1] = l2[q].y;
      HeadReduce<NC, 16>::run(l, lane);  // lane: column lane / (32 / NC)
      if (lane % (32 / NC) == 0) bars.col[warp & 3][q0 + lane / (32 / NC)] = l[0];
      ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.o_full[(c - 1) & 1], ((c - 1) >> 1) & 1));
      if (keys_any(grp, !ok)) break;
      if (key < NC) {
        const int q = q0 + key;
        const float sum = (bars.col[0][q] + bars.col[1][q]) + (bars.col[2][q] + bars.col[3][q]);
        bars.col[0][q] = w.slot >= 0 ? sum : sum != 0.f ? 1.f / sum : 0.f;
      }
      keys_sync(grp);
      tc_fence_after();
      uint32_t o[NC];
      load_cols<NC>(tmem + 2 * N + q0 + lanes, o);
      const bool whole = w.slot < 0;
      const int tok0 = w.tok0;
      if (w.bad) {  // what was cleared, for the queries that see it
        for (int blk = w.blk0; blk < w.blk1; ++blk) {
          const int i0 = w.blocks.index(blk) * kBn;
          if (!w.hides(blk)) continue;
          for (int i = i0; i < i0 + kBn && i < w.n; ++i) {
            const float z = __bfloat162float(
                ((const __nv_bfloat16 *)a.V)[(w.row0 + i) * D + key % D]);
            if (isfinite(z)) continue;
            const uint64_t see = columns_seeing(w.rows, a.shape, a.g, i) >> q0;
#pragma unroll
            for (int q = 0; q < NC; ++q)
              if (see >> q & 1) o[q] = __float_as_uint(__uint_as_float(o[q]) + z);
          }
        }
      }
      if (key < D) {
        // row q of the tile is head q % g of token q / g
        int h = q0 % a.g;
        __nv_bfloat16 *out = (__nv_bfloat16 *)a.out + key +
                             ((int64_t)(tok0 + q0 / a.g) * (a.H_kv * a.g) + w.kvh * a.g + h) * D;
        float *part =
            whole ? nullptr : (float *)part_at(a, D, blockIdx.x, w.slot, key / 4, q0) + key % 4;
        const int64_t skip = (int64_t)(a.H_kv - 1) * a.g * D;
#pragma unroll
        for (int q = 0; q < NC; ++q) {
          if (q0 + q >= used) break;
          const float x = __uint_as_float(o[q]);
          if (whole) {
            *out = __float2bfloat16_rn(x * bars.col[0][q0 + q]);
            out += D;
            if (++h == a.g) h = 0, out += skip;
          } else {
            part[q * 4] = x;
          }
        }
      }
      if (!whole && key < NC && q0 + key < used)
        *part_ml(a, D, gridDim.x, blockIdx.x, w.slot, q0 + key) =
            make_float2(bars.m[q0 + key], bars.col[0][q0 + key]);
      keys_sync(grp);  // the normalisers have been read
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&bars.o_free);
        bars.queue.done(pc);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (bars.give_up) {  // copies and products in flight end before the memory is handed on
    if (tid == 0) set_status(a.status, LG_ERR_TIMEOUT);
    linger();
    __syncthreads();
  }
  if (warp == W0 + 1) {
    tc_fence_after();
    tmem_free(tmem, kTmemCols);
  }
}

template <int D, int N>
cudaError_t launch_typed(const ChunkAttendArgs &a, int G, cudaStream_t s) {
  CUtensorMap mq, mk, mv;
  if (!make_q_map(&mq, a.q, D, a.H_kv * a.g, a.T, a.g, a.shape.tok) ||
      !make_kv_map(&mk, a.K, LG_BF16, D, a.cache_rows, kBn) ||
      !make_kv_map(&mv, a.V, LG_BF16, D, a.cache_rows, kBn))
    return cudaErrorInvalidValue;
  auto kern = chunk_attend_few_kernel<D, N>;
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              FewCfg<D, N>::kSmem));
  LG_TRY(launch_pdl(kern, G, FewCfg<D, N>::kThreads, FewCfg<D, N>::kSmem, s, mq, mk, mv, a));
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const ChunkAttendArgs &a, int G, cudaStream_t s) {
  return a.rows == 16 ? launch_typed<D, 16>(a, G, s)
         : a.rows == 32 ? launch_typed<D, 32>(a, G, s)
                        : launch_typed<D, 64>(a, G, s);
}

}  // namespace

cudaError_t launch_chunk_attend_few(const ChunkAttendArgs &a, int d, int G, cudaStream_t s) {
  return d == 128 ? launch_d<128>(a, G, s) : launch_d<64>(a, G, s);
}

}  // namespace lg
