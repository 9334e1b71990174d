// lg_chunk_attend of bf16 caches on the tensor cores (tcgen05, tensor memory, TMA).
//
// A query tile is 128 rows of the products' M: the g query heads of tok / NS consecutive new tokens
// (row r: token r / g, head r % g), copied as one box of the queries.  An item has NS tiles
// ("streams"); NS = 2 shares every key block between 256 query rows, NS = 1 is for chunks of at
// most 128 rows, whose calls are bound by reading the cache.  For each key block of 128 rows
//   S = Q K^T   (tensor memory, fp32),  P = 2^(S scale - m) (bf16, over S),  O += P V
// with the running maximum m and normaliser l in registers, one thread a row.  m follows the true
// maximum lazily: O and l are rescaled only when a maximum rose by more than 2^8, so that the
// rescaling, a pass over O in tensor memory, happens in the first blocks only; weights up to 2^8
// lose nothing in bf16 or in the fp32 sums.  P is rounded to bf16 (2^-9 of a weight, the precision
// of the values it multiplies); l sums the unrounded weights in fp32.
//
// Warps: 0-3 and 4-7 the rows of streams 0 and 1; 8 copies (TMA), 9 issues the products, 10 and 11
// clear what is not a number from the values of blocks in which some row is hidden from some query
// (0 x NaN would reach the hidden one's sums).  Those values are added again, at the end, for the
// queries that see them.
#include <cuda_bf16.h>
#include <cudaTypedefs.h>

#include "lg_chunk_attend.cuh"
#include "lg_tcgen05.cuh"

namespace lg {

namespace {

constexpr int kThreads = 384;
constexpr int kBn = 128;            // rows of a key block
constexpr float kLazy = 8.f;        // log2 of the factor that m may lag behind
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;     // S at columns 0 and 128, O at 256 and 256 + D

template <int D, int NS>
struct TcCfg {
  static constexpr int kBoxes = D / 64;                 // boxes of 64 columns
  static constexpr int kTile = kBn * D * 2;             // bytes of a key or value block
  static constexpr int kQTile = 128 * D * 2;
  static constexpr int kStages = D == 128 ? (NS == 2 ? 5 : 6) : (NS == 2 ? 10 : 12);
  static constexpr int kSmem = NS * kQTile + kStages * kTile + 1024;  // + alignment
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int ST>
struct TcBars {
  uint64_t full[ST], empty[ST];      // ring of key and value blocks
  uint64_t fixed[ST];                // what hidden rows hold is cleared
  uint64_t q_full, q_empty;
  uint64_t s_full[2], p_full[2];     // scores ready, weights ready
  uint64_t o_full[2], o_free[2];     // sums ready, sums read
  uint32_t tmem;
  volatile int bad_piece[16];        // piece i had something cleared: entry i % 16 holds i
  volatile int give_up;              // a bounded wait ran out
};

// Some row of the block from row i0 is hidden from some query of the item (or lies past the rows).
__device__ __forceinline__ bool block_hides(const TileRows &r, const ChunkShape &s, int i0) {
  if (i0 + kBn - 1 > r.first) return true;
  if (s.window == 0) return false;
  const int64_t a = plan_max(i0, s.sink);
  return a <= plan_min((int64_t)i0 + kBn - 1, (int64_t)r.last - s.window);
}

// bounded wait that also ends when another role has given up
template <typename B>
__device__ __forceinline__ bool tc_wait(B &b, uint64_t *bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  while (true) {
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (b.give_up) return false;
    if (global_ns() - t0 > kWaitLimitNs) {
      b.give_up = 1;
      return false;
    }
  }
}

// an element of a bf16 pair that is infinite or NaN: bit 15 or 31 of the result
__device__ __forceinline__ uint32_t not_numbers(uint32_t w) {
  return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

template <int D, int NS>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_attend_tc_kernel(const __grid_constant__ CUtensorMap mq,
                           const __grid_constant__ CUtensorMap mk,
                           const __grid_constant__ CUtensorMap mv, ChunkAttendArgs a) {
  using C = TcCfg<D, NS>;
  constexpr int ST = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ TcBars<ST> bars;
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sq = smem, *ring = smem + NS * C::kQTile;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int tpt = a.shape.tok / NS;  // tokens of a tile
  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 3);  // the products and both clearing warps
      mbar_init(&bars.fixed[i], 2);
    }
    mbar_init(&bars.q_full, 1);
    mbar_init(&bars.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], 4);
      mbar_init(&bars.o_full[i], 1);
      mbar_init(&bars.o_free[i], 4);
    }
    for (int i = 0; i < 16; ++i) bars.bad_piece[i] = -1;
    bars.give_up = 0;
    mbar_fence_init();
  }
  if (warp == 9) tmem_alloc(&bars.tmem, kTmemCols);
  pdl_enter();
  ChunkShare sh;
  // (its barriers also publish the mbarriers and the tensor memory's address)
  tc_fence_before();
  bool work = chunk_share<kThreads>(a, blockIdx.x, gridDim.x, sh);
  __syncthreads();
  tc_fence_after();
  work = work && sh.y0 < sh.y1;
  const uint32_t tmem = bars.tmem;
  // registers: 168 a thread at launch, 64512 in all; the rows' warps take 208, the others 88
  // (256 x 208 + 128 x 88 = 64512)
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (work && warp == 8) {
    if (lane == 0) {
      ChunkWalk w;
      uint32_t n = 0, pieces = 0;  // ring position, pieces so far
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
      for (w.start(a, sh, sh.y0); ok && !w.done(); w.next(a)) {
        if (w.blk0 == w.blk1) continue;
        const int tokens = w.tokens(a);
        const int tiles = NS == 2 && tokens > tpt ? 2 : 1;
        ok = tc_wait(bars, &bars.q_empty, (pieces & 1) ^ 1);
        if (!ok) break;
        mbar_arrive_expect_tx(&bars.q_full, tiles * C::kBoxes * tpt * a.g * 128);
        for (int s = 0; s < tiles; ++s)
#pragma unroll
          for (int x = 0; x < C::kBoxes; ++x)
            tma_box_3d(sq + s * C::kQTile + x * (128 * 128), &mq, 64 * x, w.kvh * a.g,
                       w.off + w.t * a.shape.tok + s * tpt, &bars.q_full);
        ++pieces;
        const int r0 = (int)w.row0;
        if (NS == 2) {
          for (int j = w.blk0; ok && j < w.blk1; ++j) {
            const int row = r0 + w.blocks.index(j) * kBn;
            load(&mk, row);
            load(&mv, row);
          }
        } else {  // the order in which the products take them
          load(&mk, r0 + w.blocks.index(w.blk0) * kBn);
          for (int j = w.blk0; ok && j < w.blk1; ++j) {
            if (j + 1 < w.blk1) load(&mk, r0 + w.blocks.index(j + 1) * kBn);
            load(&mv, r0 + w.blocks.index(j) * kBn);
          }
        }
      }
    }
  } else if (work && warp == 9) {
    if (lane == 0) {
      ChunkWalk w;
      uint32_t n = 0, pieces = 0, c[2] = {0, 0}, used[2] = {0, 0};
      bool ok = true;
      constexpr uint32_t kIdS = mma_idesc(128, kBn, false), kIdO = mma_idesc(128, D, true);
      uint64_t dq[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) dq[s] = smem_desc(smem_addr(sq + s * C::kQTile), 16, 1024);
      auto stage = [&](uint32_t i) { return smem_addr(ring + i % ST * C::kTile); };
      auto wait_full = [&](uint32_t i) {
        ok = ok && tc_wait(bars, &bars.full[i % ST], (i / ST) & 1);
      };
      // S (buffer b) = Q (tile s) K^T with the key block at ring position i
      auto qk = [&](int s, int b, uint32_t i) {
        if (!ok) return;
        tc_fence_after();
        const uint64_t dk = smem_desc(stage(i), 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t at = (uint64_t)(((k / 4) * (128 * 128) + (k % 4) * 32) >> 4);
          tc_mma_ss(tmem + b * 128, dq[s] + at, dk + at, kIdS, k > 0);
        }
        tc_commit(&bars.s_full[b]);
      };
      // O (tile s) += P (buffer b) V with the value block at ring position i
      auto pv = [&](int s, int b, uint32_t i, bool add) {
        if (!ok) return;
        tc_fence_after();
        const uint64_t dv = smem_desc(stage(i), kBn * 128, 1024);
#pragma unroll
        for (int k = 0; k < kBn / 16; ++k)
          tc_mma_ts(tmem + kColO + s * D, tmem + b * 128 + k * 8, dv + (uint64_t)(k * 2048 >> 4),
                    kIdO, add || k > 0);
      };
      auto wait_v = [&](uint32_t i, bool hides) {
        wait_full(i);
        if (hides) ok = ok && tc_wait(bars, &bars.fixed[i % ST], (i / ST) & 1);
      };
      for (w.start(a, sh, sh.y0); ok && !w.done(); w.next(a)) {
        if (w.blk0 == w.blk1) continue;
        const int blocks = w.blk1 - w.blk0;
        ok = tc_wait(bars, &bars.q_full, pieces & 1);
        ++pieces;
        if (NS == 2) {
          const bool two = w.tokens(a) > tpt;
          wait_full(n);
          qk(0, 0, n);
          if (two) qk(NS - 1, 1, n);
          if (!ok) break;
          tc_commit(&bars.empty[n % ST]);
          if (blocks == 1) tc_commit(&bars.q_empty);
          for (int j = 0; ok && j < blocks; ++j) {
            const bool more = j + 1 < blocks;
            const uint32_t iv = n + 2 * j + 1, ik = iv + 1;
            wait_v(iv, block_hides(w.rows, a.shape, w.blocks.index(w.blk0 + j) * kBn));
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              if (s == 1 && !two) break;
              if (j == 0) {
                ok = ok && tc_wait(bars, &bars.o_free[s], (used[s] & 1) ^ 1);
                ++used[s];
              }
              ok = ok && tc_wait(bars, &bars.p_full[s], c[s] & 1);
              ++c[s];
              pv(s % NS, s, iv, j > 0);
              if (more) {
                if (s == 0) wait_full(ik);
                qk(s % NS, s, ik);
              } else if (ok) {
                tc_commit(&bars.o_full[s]);
              }
            }
            if (!ok) break;
            tc_commit(&bars.empty[iv % ST]);
            if (more) {
              tc_commit(&bars.empty[ik % ST]);
              if (j + 2 == blocks) tc_commit(&bars.q_empty);
            }
          }
        } else {
          // scores of the next block are formed while this one's weights are; c[0] counts blocks
          auto k_at = [&](int j) { return n + (j == 0 ? 0 : 2 * j - 1); };
          auto first = [&](int j) {
            wait_full(k_at(j));
            qk(0, (c[0] + j) & 1, k_at(j));
            if (!ok) return;
            tc_commit(&bars.empty[k_at(j) % ST]);
            if (j + 1 == blocks) tc_commit(&bars.q_empty);
          };
          first(0);
          for (int j = 0; ok && j < blocks; ++j) {
            if (j + 1 < blocks) first(j + 1);
            const uint32_t iv = n + (j + 1 < blocks ? 2 * j + 2 : 2 * j + 1), cj = c[0] + j;
            wait_v(iv, block_hides(w.rows, a.shape, w.blocks.index(w.blk0 + j) * kBn));
            if (j == 0) {
              ok = ok && tc_wait(bars, &bars.o_free[0], (used[0] & 1) ^ 1);
              ++used[0];
            }
            ok = ok && tc_wait(bars, &bars.p_full[cj & 1], (cj >> 1) & 1);
            pv(0, cj & 1, iv, j > 0);
            if (!ok) break;
            tc_commit(&bars.o_full[0]);
            tc_commit(&bars.empty[iv % ST]);
          }
          c[0] += blocks;
        }
        n += 2 * blocks;
      }
    }
  } else if (work && warp >= 10) {
    ChunkWalk w;
    uint32_t n = 0;
    int piece = 0;
    bool ok = true;
    for (w.start(a, sh, sh.y0); ok && !w.done(); w.next(a)) {
      if (w.blk0 == w.blk1) continue;
      const int blocks = w.blk1 - w.blk0;
      for (int i = 0; ok && i < 2 * blocks; ++i, ++n) {
        // the i-th copy of the piece: a key block, or the values of block j
        int j = -1;
        if (NS == 2) {
          if (i & 1) j = i >> 1;
        } else if (i == 2 * blocks - 1) {
          j = blocks - 1;
        } else if (i >= 2 && !(i & 1)) {
          j = i / 2 - 1;
        }
        ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.full[n % ST], (n / ST) & 1));
        if (!ok) break;
        const int i0 = j < 0 ? 0 : w.blocks.index(w.blk0 + j) * kBn;
        if (j >= 0 && block_hides(w.rows, a.shape, i0)) {
          uint4 *v = (uint4 *)(ring + n % ST * C::kTile);
          bool bad = false;
          for (int e = tid - 320; e < C::kTile / 16; e += 64) {
            uint4 u = v[e];
            uint32_t *uw = (uint32_t *)&u;
            if (not_numbers(u.x) | not_numbers(u.y) | not_numbers(u.z) | not_numbers(u.w)) {
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const uint32_t b = not_numbers(uw[x]);
                uw[x] &= (b & 0x8000u ? 0u : 0xffffu) | (b & 0x80000000u ? 0u : 0xffff0000u);
              }
              v[e] = u;
              bad |= i0 + e / 8 % kBn < w.q.n;
            }
          }
          if (bad) bars.bad_piece[piece & 15] = piece;  // (at most ST / 2 + 1 pieces ahead)
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (lane == 0) {
          mbar_arrive(&bars.fixed[n % ST]);
          mbar_arrive(&bars.empty[n % ST]);
        }
      }
      ++piece;
    }
  }
  } else {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
  if (work && (NS == 2 || warp < 4)) {
    const int s = warp >> 2;                  // stream
    const int r = tid & 127;                  // row of the tile
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // lane 32 (warp % 4) in bits 16..
    const uint32_t to = tmem + kColO + (NS == 2 ? s * D : 0) + lanes;
    const int H_q = a.H_kv * a.g;
    const int j_tok = s * tpt + r / a.g;      // token of the row in the item
    ChunkWalk w;
    uint32_t c = 0, pieces = 0;               // blocks and pieces of this stream so far
    int piece = 0;
    bool ok = true;
    for (w.start(a, sh, sh.y0); ok && !w.done(); w.next(a)) {
      if (w.blk0 == w.blk1) continue;
      const int used = (min(w.tokens(a), (s + 1) * tpt) - s * tpt) * a.g;  // rows that are queries
      if (used <= 0) {
        ++piece;
        continue;
      }
      const bool idle = (warp & 3) * 32 >= used;  // no row of this warp is one
      const int qrow = w.rows.first + j_tok;
      float m = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f);
      for (int blk = w.blk0; blk < w.blk1; ++blk, ++c) {
        const int b = NS == 2 ? s : (int)(c & 1);
        const uint32_t par = NS == 2 ? c & 1 : (c >> 1) & 1;
        const uint32_t ts = tmem + b * 128 + lanes;
        ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.s_full[b], par));
        if (!ok) break;
        if (!idle) {
          tc_fence_after();
          uint32_t u[kBn];
#pragma unroll
          for (int x = 0; x < kBn; x += 32) tmem_load32(ts + x, u + x);
          tmem_wait_load();
          float *v = (float *)u;
          const int i0 = w.blocks.index(blk) * kBn;
          if (block_hides(w.rows, a.shape, i0)) {
            const int lo = a.shape.window ? (int)plan_max((int64_t)qrow - a.shape.window, -1) : -1;
#pragma unroll
            for (int x = 0; x < kBn; ++x) {
              const int i = i0 + x;
              if (i > qrow || (i <= lo && i >= a.shape.sink)) v[x] = -INFINITY;
            }
          }
          float mx = v[0];
#pragma unroll
          for (int x = 1; x < kBn; ++x) mx = fmaxf(mx, v[x]);
          mx *= a.qscale;
          const bool rise = mx > m + kLazy || m == -INFINITY;
          if (__any_sync(0xffffffffu, rise)) {
            const float m1 = rise ? fmaxf(m, mx) : m;
            const float f = rise ? (m == -INFINITY ? 0.f : exp2_fast(m - m1)) : 1.f;
            m = m1;
            l2.x *= f;
            l2.y *= f;
            if (blk > w.blk0) {
              // (NS = 2: the scores were formed after the previous block's sums)
              if (NS == 1) {
                ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.o_full[0], (c - 1) & 1));
                if (!ok) break;
                tc_fence_after();
              }
#pragma unroll
              for (int x = 0; x < D; x += 32) {
                uint32_t o[32];
                tmem_load32(to + x, o);
                tmem_wait_load();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_store32(to + x, o);
              }
            }
          }
          const float nb = m == -INFINITY ? 0.f : -m;
          const float2 sc = make_float2(a.qscale, a.qscale), mb = make_float2(nb, nb);
#pragma unroll
          for (int x = 0; x < kBn; x += 64) {
            uint32_t p[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float2 z = __ffma2_rn(make_float2(v[x + 2 * e], v[x + 2 * e + 1]), sc, mb);
              z.x = exp2_fast(z.x);
              z.y = exp2_fast(z.y);
              l2 = __fadd2_rn(l2, z);
              const __nv_bfloat162 h = __floats2bfloat162_rn(z.x, z.y);
              p[e] = *(const uint32_t *)&h;
            }
            tmem_store32(ts + x / 2, p);
          }
          tmem_wait_store();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full[b]);
      }
      if (!ok) break;
      ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.o_full[NS == 2 ? s : 0],
                                           NS == 2 ? pieces & 1 : (c - 1) & 1));
      if (!ok) break;
      ++pieces;
      tc_fence_after();
      if (!idle) {
        const float l = l2.x + l2.y;
        const bool whole = w.whole(), bad = bars.bad_piece[piece & 15] == piece;
        const float inv = whole ? (l != 0.f ? 1.f / l : 0.f) : 1.f;
        const int64_t dst =
            ((int64_t)(w.off + w.t * a.shape.tok + j_tok) * H_q + w.kvh * a.g + r % a.g) * D;
        const int pr = s * tpt * a.g + r;
#pragma unroll 1
        for (int x = 0; x < D; x += 32) {
          uint32_t o[32];
          tmem_load32(to + x, o);
          tmem_wait_load();
          if (r < used) {
          if (bad) {  // what was cleared and this query sees
            for (int blk = w.blk0; blk < w.blk1; ++blk) {
              const int i0 = w.blocks.index(blk) * kBn;
              if (!block_hides(w.rows, a.shape, i0)) continue;
              for (int i = i0; i < i0 + kBn && i < w.q.n; ++i) {
                if (!row_sees(w.rows, a.shape, qrow, i)) continue;
                const __nv_bfloat16 *vr = (const __nv_bfloat16 *)a.V + (w.row0 + i) * D + x;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const float z = __bfloat162float(vr[e]);
                  if (!isfinite(z)) o[e] = __float_as_uint(__uint_as_float(o[e]) + z);
                }
              }
            }
          }
          if (whole) {
            uint32_t h[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const __nv_bfloat162 z = __floats2bfloat162_rn(__uint_as_float(o[2 * e]) * inv,
                                                             __uint_as_float(o[2 * e + 1]) * inv);
              h[e] = *(const uint32_t *)&z;
            }
            uint4 *p = (uint4 *)((__nv_bfloat16 *)a.out + dst + x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              p[e] = make_uint4(h[4 * e], h[4 * e + 1], h[4 * e + 2], h[4 * e + 3]);
          } else {
            uint4 *p = (uint4 *)(part_row(a, D, blockIdx.x, w.slot(), pr) + x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              p[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
          }
          __syncwarp();  // every lane loads the next columns together
        }
        if (!whole && r < used)
          *part_ml(a, D, gridDim.x, blockIdx.x, w.slot(), pr) = make_float2(m, l);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.o_free[NS == 2 ? s : 0]);
      ++piece;
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
  if (warp == 9) {
    tc_fence_after();
    tmem_free(tmem, kTmemCols);
  }
}

// the queries [T][H_q][d] in boxes of 64 columns, g heads and `tokens` tokens
bool make_q_map(CUtensorMap *m, const void *q, int d, int H_q, int T, int g, int tokens) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)H_q, (cuuint64_t)T};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)d * 2 * H_q};
  cuuint32_t box[3] = {64, (cuuint32_t)g, (cuuint32_t)tokens};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(q), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int NS>
cudaError_t launch_typed(const ChunkAttendArgs &a, int G, cudaStream_t s) {
  CUtensorMap mq, mk, mv;
  if (!make_q_map(&mq, a.q, D, a.H_kv * a.g, a.T, a.g, a.shape.tok / NS) ||
      !make_kv_map(&mk, a.K, LG_BF16, D, a.cache_rows, kBn) ||
      !make_kv_map(&mv, a.V, LG_BF16, D, a.cache_rows, kBn))
    return cudaErrorInvalidValue;
  auto kern = chunk_attend_tc_kernel<D, NS>;
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              TcCfg<D, NS>::kSmem));
  LG_TRY(launch_pdl(kern, G, kThreads, TcCfg<D, NS>::kSmem, s, mq, mk, mv, a));
  return cudaGetLastError();
}

}  // namespace

ChunkGrid chunk_grid_tc(int g, int max_new) {
  ChunkGrid r;
  // two tiles an item where some sequence fills more than one
  const int tiles = (int64_t)max_new > 128 / g ? 2 : 1;
  r.ctas = 152;
  r.rows = 128 * tiles;
  r.tok = 128 / g * tiles;
  r.bn = kBn;
  return r;
}

cudaError_t launch_chunk_attend_tc(const ChunkAttendArgs &a, int d, int G, cudaStream_t s) {
  if (a.rows == 256)
    return d == 128 ? launch_typed<128, 2>(a, G, s) : launch_typed<64, 2>(a, G, s);
  return d == 128 ? launch_typed<128, 1>(a, G, s) : launch_typed<64, 1>(a, G, s);
}

}  // namespace lg
