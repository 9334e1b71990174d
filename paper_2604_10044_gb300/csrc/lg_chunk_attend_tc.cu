// lg_chunk_attend of bf16 caches on the tensor cores (tcgen05, tensor memory, TMA).
//
// A query tile is 128 rows of the products' M: the g query heads of tok / 2 consecutive new tokens
// (row r: token r / g, head r % g), copied as one box of the queries.  An item has two tiles
// ("streams"), so that every key block serves 256 query rows and the products of one stream run
// while the other's weights are formed.  For each key block of 128 rows (64 for heads of 64 elements)
//   S = Q K^T   (tensor memory, fp32),  P = 2^(S scale - m) (bf16, over S),  O += P V
// with the running maximum m and normaliser l in registers, one thread a row.  m follows the true
// maximum lazily: O and l are rescaled only when a maximum rose by more than 2^8, so that the
// rescaling, a pass over O in tensor memory, happens in the first blocks only; weights up to 2^8
// lose nothing in bf16 or in the fp32 sums.  P is rounded to bf16 (half a step, 2^-8 of a weight at
// most: the precision of the values it multiplies); l sums the unrounded weights in fp32.
//
// Heads of 128 elements: the products of a stream take as long as its weights, S and O of two streams
// fill the tensor memory, and a stream's next scores follow its sums.  Heads of 64: half the products
// for the same weights, so the weights are the bound; blocks of 64 keys leave room for two buffers of
// S a stream, scores are formed two blocks ahead, and the rows' warps never wait for them.  (Products
// with N = 64 read the queries as often as the keys, 1.5 x the time of N = 128: too slow for 128.)
//
// Warps: 0-3 and 4-7 the rows of streams 0 and 1; 8 walks along the work and copies (TMA), 9 and 10
// issue the products of a stream each, 11 clears what is not a number from the values of blocks in
// which some row is hidden from some query (0 x NaN would reach the hidden one's sums).  Those values
// are added again, at the end, for the queries that see them.
#include "lg_chunk_tc.cuh"

namespace lg {
namespace {

constexpr int kThreads = 384;
constexpr float kLazy = 8.f;        // log2 of the factor that m may lag behind
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;     // S below column 256 (a stream's buffers together), O from there

template <int D>
struct TcCfg {
  static constexpr int kBn = D == 128 ? 128 : 64;       // rows of a key block
  static constexpr int kBufs = 128 / kBn;               // buffers of S of a stream
  static constexpr int kBoxes = D / 64;                 // boxes of 64 columns
  static constexpr int kTile = kBn * D * 2;             // bytes of a key or value block
  static constexpr int kQTile = 128 * D * 2;
  static constexpr int kStages = D == 128 ? 5 : 16;
  static constexpr int kSmem = 2 * kQTile + kStages * kTile + 1024;  // + alignment
};

template <int ST>
struct TcBars {
  uint64_t full[ST], empty[ST];      // ring of key and value blocks
  uint64_t fixed[ST];                // what hidden rows hold is cleared
  uint64_t q_full[2], q_empty;       // a stream's queries, of the pieces that it has part in; all read
  // of stream s and buffer b, at 2 s + b: scores ready, half of and all weights ready, sums ready (with
  // one buffer: the piece's)
  uint64_t s_full[4], p_half[4], p_full[4], o_full[4];
  uint64_t o_free[2];                // sums read
  uint64_t turn[2];                  // the stream's products are next
  TcQueue queue;
  uint32_t tmem;
  volatile int give_up;              // a bounded wait ran out
};

// Lanes that differ in bit B of their number exchange: the lower one its b for the upper one's a.
template <int B>
__device__ __forceinline__ void swap_pieces(uint4 &a, uint4 &b, int lane) {
  const bool up = (lane & B) != 0;
  uint32_t *x = (uint32_t *)&a, *y = (uint32_t *)&b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? x[i] : y[i], B);
    if (up)
      x[i] = got;
    else
      y[i] = got;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_attend_tc_kernel(const __grid_constant__ CUtensorMap mq,
                           const __grid_constant__ CUtensorMap mk,
                           const __grid_constant__ CUtensorMap mv, ChunkAttendArgs a) {
  using C = TcCfg<D>;
  constexpr int ST = C::kStages, kBn = C::kBn, NB = C::kBufs;
  extern __shared__ uint8_t smem_raw[];
  __shared__ TcBars<ST> bars;
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sq = smem, *ring = smem + 2 * C::kQTile;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int tpt = a.shape.tok / 2;  // tokens of a tile
  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 3);  // both streams' products and the clearing warp
      mbar_init(&bars.fixed[i], 1);
    }
    mbar_init(&bars.q_empty, 2);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_half[i], 4);
      mbar_init(&bars.p_full[i], 4);
      mbar_init(&bars.o_full[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.q_full[i], 1);
      mbar_init(&bars.o_free[i], 4);
      mbar_init(&bars.turn[i], 1);
    }
    bars.queue.init(11);               // the products' two warps, the clearing one, eight of rows
    bars.give_up = 0;
    mbar_fence_init();
  }
  if (warp == 9) tmem_alloc(&bars.tmem, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_enter();
  const uint32_t tmem = bars.tmem;

  // registers: 168 a thread at launch, 64512 in all; the rows' warps take 208, the others 88
  // (256 x 208 + 128 x 88 = 64512)
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8) {
      ChunkShare sh;
      const bool work = chunk_share<false>(a, blockIdx.x, gridDim.x, sh);
      if (lane == 0) {
        // Heads of 64 keep the walk in shared memory (two prompts of 8192, 32/8 heads: 557 us, 585
        // in registers), heads of 128 in registers (16 x 512 new rows: 78.7 us, 79.9 in shared
        // memory).
        __shared__ ChunkWalk<false> far;
        ChunkWalk<false> near;
        ChunkWalk<false> &w = D == 64 ? far : near;
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
        if (work) w.start(a, sh);
        put_cut(a, D, gridDim.x, blockIdx.x, work, sh, w);
        for (; work && ok && !w.done(); w.next(a)) {
          if (w.blk0 == w.blk1) continue;
          const int tiles = w.tokens(a) > tpt ? 2 : 1;
          ok = bars.queue.put(bars, pieces, w, a) &&
               tc_wait(bars, &bars.q_empty, (pieces & 1) ^ 1);
          if (!ok) break;
          for (int s = 0; s < tiles; ++s) {
            mbar_arrive_expect_tx(&bars.q_full[s], C::kBoxes * tpt * a.g * 128);
#pragma unroll
            for (int x = 0; x < C::kBoxes; ++x)
              tma_box_3d(sq + s * C::kQTile + x * (128 * 128), &mq, 64 * x, w.kvh * a.g,
                         w.off + w.t * a.shape.tok + s * tpt, &bars.q_full[s]);
          }
          ++pieces;
          // keys NB blocks ahead of the values, as the products take them
          auto row = [&](int j) { return (int)w.row0 + w.blocks.index(j) * kBn; };
          for (int j = w.blk0; ok && j < w.blk1 && j < w.blk0 + NB; ++j) load(&mk, row(j));
          for (int j = w.blk0; ok && j < w.blk1; ++j) {
            load(&mv, row(j));
            if (j + NB < w.blk1) load(&mk, row(j + NB));
          }
        }
        if (ok) bars.queue.end(bars, pieces);
      }
    } else if (warp <= 10) {
      // One warp a stream: what surrounds the products (waits, commits) takes as long as the products
      // of one stream, and one warp for both kept the tensor cores waiting (56 % busy).  They take
      // turns, a stream's sums and next scores at a time: products that both have in flight finish
      // together, then both streams form weights and the tensor cores stand still.
      const int s = warp - 9;
      const bool one = elect_one();
      uint32_t n = 0, c = 0, mine = 0;  // ring position; blocks and pieces of the stream
      uint32_t turns = 0;               // blocks that both streams had
      bool ok = true;
      constexpr uint32_t kIdS = mma_idesc(128, kBn, false, false);
      constexpr uint32_t kIdO = mma_idesc(128, D, false, true);
      const uint32_t ts0 = tmem + s * 128, to = tmem + kColO + s * D;
      const uint32_t q_lo = desc_lo(smem_addr(sq + s * C::kQTile), 16);
      const uint32_t k_lo = desc_lo(smem_addr(ring), 16), v_lo = desc_lo(smem_addr(ring), kBn * 128);
      auto wait_full = [&](uint32_t i) {
        ok = ok && tc_wait_warp(bars, &bars.full[i % ST], (i / ST) & 1);
      };
      // S = Q K^T into buffer b with the key block at ring position i (which has arrived)
      auto qk = [&](uint32_t b, uint32_t i, bool last) {
        const uint32_t k0 = k_lo + i % ST * (C::kTile >> 4);
        if (one) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            tc_mma_ss(ts0 + b * kBn, q_lo + (((k / 4) * (128 * 128) + (k % 4) * 32) >> 4),
                      k0 + (((k / 4) * (kBn * 128) + (k % 4) * 32) >> 4), kIdS, k > 0);
          }
          tc_commit(&bars.s_full[2 * s + b]);
          tc_commit(&bars.empty[i % ST]);
          if (last) tc_commit(&bars.q_empty);
        }
      };
      for (uint32_t pc = 0;; ++pc) {
        ok = bars.queue.wait(bars, pc);
        if (!ok) break;
        const TcPiece &p = bars.queue.at(pc);
        const int blk1 = uniform(p.blk1);
        if (blk1 < 0) break;
        const int blocks = blk1 - uniform(p.blk0);
        const int open0 = uniform(p.open0 - p.blk0), open1 = uniform(p.open1 - p.blk0);
        const bool two = uniform(p.tokens) > tpt, active = s == 0 || two;
        __syncwarp();
        if (one) bars.queue.done(pc);
        if (!active) {  // the other stream's blocks pass
          for (int i = 0; ok && i < 2 * blocks; ++i, ++n) {
            wait_full(n);
            if (ok && one) mbar_arrive(&bars.empty[n % ST]);
          }
          if (!ok) break;
          if (one) mbar_arrive(&bars.q_empty);
          continue;
        }
        ok = tc_wait_warp(bars, &bars.q_full[s], mine & 1);
        const int ahead = blocks < NB ? blocks : NB;
        for (int i = 0; i < ahead; ++i) {
          wait_full(n + i);
          if (!ok) break;
          tc_fence_after();
          qk((c + i) % NB, n + i, i + 1 == blocks);
        }
        ok = ok && tc_wait_warp(bars, &bars.o_free[s], (mine & 1) ^ 1);
        ++mine;
        for (int j = 0; ok && j < blocks; ++j, ++c) {
          // (value block j follows the keys ahead of it and j pairs, or what pairs there are)
          const uint32_t iv = n + ahead + j + (j < blocks - ahead ? j : blocks - ahead);
          const uint32_t b = c % NB, par = (c / NB) & 1, ts = ts0 + b * kBn;
          // The next keys, and the values, or, where the block hides rows, their clearing.  A copy's
          // arrival, the values' own or a later one's, says that the ring's slot has been through the
          // clearing warp before, and so which phase of `fixed` the parity means.
          const bool last = j + NB >= blocks;
          wait_full(last ? iv : iv + 1);
          if (j < open0 || j >= open1)
            ok = ok && tc_wait_warp(bars, &bars.fixed[iv % ST], (iv / ST) & 1);
          else if (!last)
            wait_full(iv);
          ok = ok && tc_wait_warp(bars, &(NB == 1 ? bars.p_half : bars.p_full)[2 * s + b], par);
          if (NB == 1 && two) ok = ok && tc_wait_warp(bars, &bars.turn[s], (turns & 1) ^ (s ^ 1));
          if (!ok) break;
          tc_fence_after();
          // O += P V (one buffer: the block's first half while the second one's weights are formed)
          const uint32_t v0 = v_lo + iv % ST * (C::kTile >> 4);
          auto pv = [&](int k0) {
            if (one) {
#pragma unroll
              for (int k = 0; k < kBn / 32; ++k)
                tc_mma_ts(to, ts + (k0 + k) * 8, v0 + (k0 + k) * (2048 >> 4), kIdO,
                          j > 0 || k0 + k > 0);
            }
          };
          pv(0);
          if (NB == 1) {
            ok = tc_wait_warp(bars, &bars.p_full[2 * s + b], par);
            if (!ok) break;
            tc_fence_after();
          }
          pv(kBn / 32);
          if (one && (NB == 2 || j + 1 == blocks)) tc_commit(&bars.o_full[2 * s + b]);
          if (j + NB < blocks) qk(b, iv + 1, j + NB + 1 == blocks);
          if (NB == 1 && two) {
            if (one) mbar_arrive(&bars.turn[s ^ 1]);
            ++turns;
          }
          if (one) tc_commit(&bars.empty[iv % ST]);
        }
        if (!ok) break;
        n += 2 * blocks;
      }
    } else {
      uint32_t n = 0;
      bool ok = true;
      for (uint32_t pc = 0; ok; ++pc) {
        ok = bars.queue.wait(bars, pc);
        if (!ok) break;
        TcPiece &p = bars.queue.at(pc);
        if (p.blk1 < 0) break;
        const int blocks = p.blk1 - p.blk0;
        const int ahead = blocks < NB ? blocks : NB;
        for (int i = 0; i < 2 * blocks; ++i, ++n) {
          ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.full[n % ST], (n / ST) & 1));
          if (!ok) break;
          // the i-th copy of the piece: keys ahead, then values and keys in turn, then values
          const int x = i - ahead, pairs = blocks - ahead;
          const int j = x < 0 ? -1 : x >= 2 * pairs ? x - pairs : x & 1 ? -1 : x >> 1;
          if (j >= 0 && p.hides(p.blk0 + j)) {
            const int i0 = p.blocks.index(p.blk0 + j) * kBn;
            if (clear_block<C::kTile, kBn>(ring + n % ST * C::kTile, i0, p.n, lane, 32)) p.bad = 1;
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
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int s = warp >> 2;                  // stream
    const int r = tid & 127;                  // row of the tile
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // lane 32 (warp % 4) in bits 16..
    const uint32_t to = tmem + kColO + s * D + lanes;
    const int j_tok = s * tpt + r / a.g, head = r % a.g;  // the row's token in the item, and its head
    uint32_t c = 0, mine = 0;                 // blocks and pieces of this stream so far
    bool ok = true;
    for (uint32_t pc = 0; ok; ++pc) {
      ok = bars.queue.wait(bars, pc);
      if (!ok) break;
      const TcPiece &p = bars.queue.at(pc);
      if (p.blk1 < 0) break;
      const int used = (min(p.tokens, (s + 1) * tpt) - s * tpt) * a.g;  // rows that are queries
      if (used > 0) {
        const bool idle = (warp & 3) * 32 >= used;  // no row of this warp is one
        const int qrow = p.rows.first + j_tok;
        const int hid = a.shape.window ? max(qrow - a.shape.window, -1) : -1;
        float m = -INFINITY;
        float2 l2 = make_float2(0.f, 0.f);
        const int blk0 = p.blk0, blk1 = p.blk1, open0 = p.open0, open1 = p.open1;
        const bool alive = r < used;
        for (int blk = blk0; blk < blk1; ++blk, ++c) {
          const bool hides = blk < open0 || blk >= open1;
          const uint32_t b = c % NB, ts = tmem + s * 128 + b * kBn + lanes;
          ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.s_full[2 * s + b], (c / NB) & 1));
          if (!ok) break;
          if (!idle) {
            tc_fence_after();
            uint32_t u[kBn];
            float *v = (float *)u;
#pragma unroll
            for (int x = 0; x < kBn; x += 32) tmem_load32(ts + x, u + x);
            tmem_wait_load();
            if (hides) {
              const int i0 = p.blocks.index(blk) * kBn;
#pragma unroll
              for (int x = 0; x < kBn; x += 32) {
                const uint32_t see = rows_seen(a.shape, qrow, hid, i0 + x);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (!(see >> e & 1)) v[x + e] = -INFINITY;
              }
            }
            float mx[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) mx[x] = fmaxf(v[x], v[x + 4]);
#pragma unroll
            for (int e = 8; e < kBn; e += 8)
#pragma unroll
              for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], v[e + x], v[e + x + 4]);
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.qscale;
            // (rows that are no query may hold anything, a NaN in every block too)
            const bool rise = alive && (top > m + kLazy || m == -INFINITY);
            if (__any_sync(0xffffffffu, rise)) {
              if (NB == 2 && blk > blk0) {
                ok = __all_sync(0xffffffffu, tc_wait(bars, &bars.o_full[2 * s + (c - 1) % NB],
                                                     ((c - 1) / NB) & 1));
                if (!ok) break;
                tc_fence_after();
              }
              const float m1 = rise ? fmaxf(m, top) : m;
              const float f = rise ? (m == -INFINITY ? 0.f : exp2_fast(m - m1)) : 1.f;
              m = m1;
              l2.x *= f;
              l2.y *= f;
              if (blk > blk0) {  // (with one buffer the scores followed the previous block's sums)
#pragma unroll 1
                for (int x = 0; x < D; x += 16) {
                  uint32_t o[16];
                  tmem_load16(to + x, o);
                  tmem_wait_load();
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                  tmem_store16(to + x, o);
                }
              }
            }
            const float nb = m == -INFINITY ? 0.f : -m;
            const float2 sc = make_float2(a.qscale, a.qscale), mb = make_float2(nb, nb);
#pragma unroll
            for (int x = 0; x < kBn; x += 32) {
              uint32_t h[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                float2 z = __ffma2_rn(make_float2(v[x + 2 * e], v[x + 2 * e + 1]), sc, mb);
                z.x = exp2_fast(z.x);
                z.y = exp2_fast(z.y);
                l2 = __fadd2_rn(l2, z);
                const __nv_bfloat162 y = __floats2bfloat162_rn(z.x, z.y);
                h[e] = *(const uint32_t *)&y;
              }
              tmem_store16(ts + x / 2, h);  // over scores that have been read
              if (NB == 1 && x == kBn / 2 - 32) {
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.p_half[2 * s + b]);
              }
            }
            tmem_wait_store();
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) {
            if (NB == 1 && idle) mbar_arrive(&bars.p_half[2 * s + b]);
            mbar_arrive(&bars.p_full[2 * s + b]);
          }
        }
        if (!ok) break;
        // (two buffers: the last block's sums; one: the piece's)
        ok = __all_sync(0xffffffffu, NB == 2 ? tc_wait(bars, &bars.o_full[2 * s + (c - 1) % NB],
                                                       ((c - 1) / NB) & 1)
                                             : tc_wait(bars, &bars.o_full[2 * s], mine & 1));
        if (!ok) break;
        ++mine;
        tc_fence_after();
        if (!idle) {
          const float l = l2.x + l2.y;
          const bool whole = p.slot < 0, bad = p.bad;
          const float inv = whole ? (l != 0.f ? 1.f / l : 0.f) : 1.f;
          const int pr = s * tpt * a.g + r;
          // results leave in stretches of 64 bytes a row: lane 4 i + j writes the j-th 16 bytes of rows
          // 4 i .. 4 i + 3 (a lane writing its own row would touch 32 lines an instruction)
          int64_t dst[4];
          {
            const int64_t own =
                r < used ? ((int64_t)(p.tok0 + j_tok) * (a.H_kv * a.g) + p.kvh * a.g + head) * D
                         : -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = __shfl_sync(0xffffffffu, own, (lane & 28) + i);
          }
#pragma unroll 1
          for (int x = 0; x < D; x += 32) {
            uint32_t o[32];
            tmem_load32(to + x, o);
            tmem_wait_load();
            if (bad && r < used) {  // what was cleared and this query sees
              for (int blk = blk0; blk < blk1; ++blk) {
                const int i0 = p.blocks.index(blk) * kBn;
                if (!p.hides(blk)) continue;
                for (int i = i0; i < i0 + kBn && i < p.n; ++i) {
                  if (!row_sees(p.rows, a.shape, qrow, i)) continue;
                  const __nv_bfloat16 *vr = (const __nv_bfloat16 *)a.V + (p.row0 + i) * D + x;
#pragma unroll
                  for (int e = 0; e < 32; ++e) {
                    const float z = __bfloat162float(vr[e]);
                    if (!isfinite(z)) o[e] = __float_as_uint(__uint_as_float(o[e]) + z);
                  }
                }
              }
            }
            __syncwarp();
            if (whole) {
              uint4 h[4];  // the row's four 16-byte pieces
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const __nv_bfloat162 z = __floats2bfloat162_rn(
                    __uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
                ((uint32_t *)h)[e] = *(const uint32_t *)&z;
              }
              // transposed among four lanes: piece i of this row <-> piece of row i
              swap_pieces<1>(h[0], h[1], lane);
              swap_pieces<1>(h[2], h[3], lane);
              swap_pieces<2>(h[0], h[2], lane);
              swap_pieces<2>(h[1], h[3], lane);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (dst[i] >= 0)
                  *(uint4 *)((__nv_bfloat16 *)a.out + dst[i] + x + 8 * (lane & 3)) = h[i];
            } else if (r < used) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *(uint4 *)part_at(a, D, blockIdx.x, p.slot, x / 4 + e, pr) =
                    make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            }
            __syncwarp();  // every lane loads the next columns together
          }
          if (!whole && r < used)
            *part_ml(a, D, gridDim.x, blockIdx.x, p.slot, pr) = make_float2(m, l);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.o_free[s]);
      }
      __syncwarp();
      if (lane == 0) bars.queue.done(pc);
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

template <int D>
cudaError_t launch_typed(const ChunkAttendArgs &a, int G, cudaStream_t s) {
  CUtensorMap mq, mk, mv;
  if (!make_q_map(&mq, a.q, D, a.H_kv * a.g, a.T, a.g, a.shape.tok / 2) ||
      !make_kv_map(&mk, a.K, LG_BF16, D, a.cache_rows, TcCfg<D>::kBn) ||
      !make_kv_map(&mv, a.V, LG_BF16, D, a.cache_rows, TcCfg<D>::kBn))
    return cudaErrorInvalidValue;
  auto kern = chunk_attend_tc_kernel<D>;
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, TcCfg<D>::kSmem));
  LG_TRY(launch_pdl(kern, G, kThreads, TcCfg<D>::kSmem, s, mq, mk, mv, a));
  return cudaGetLastError();
}

}  // namespace

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

ChunkGrid chunk_grid_tc(int d, int g, int max_new) {
  ChunkGrid r;
  const int64_t rows = (int64_t)max_new * g;
  // few rows: the kernel that takes them as the products' N (lg_chunk_attend_few.cu)
  r.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 256;
  r.ctas = 152;  // one an SM of a GB300 (on fewer SMs the others follow: no CTA waits for another)
  r.tok = r.rows == 256 ? 128 / g * 2 : r.rows / g;
  r.bn2 = r.rows == 256 && d == 64 ? 6 : 7;  // TcCfg<D>::kBn
  return r;
}

// How many lines (lg_chunk_plan.cuh): on one, a CTA comes back to a kv-head's rows when all CTAs
// have walked a tile's rows of theirs; past the L2's 126 MB it reads them from HBM again.  At 8 x
// 512 new tokens over 8192 rows, 32/8 heads of 128, one, two, four and eight lines take 378, 352,
// 338 and 330 us; two prompts of 12288 1682, 1659, 1625 and 1586.  Where the rows of the tiles under
// way fit the L2 there is nothing to gain: one prompt of 1024 takes 21.3 us on one line and 24.2 on
// eight, eight of 2048 under a window of 1024 take 142 and 141.
int chunk_lanes2(const ChunkAttendArgs &a, int d, int G) {
  int64_t rows = a.max_len;
  if (a.shape.window) rows = plan_min(rows, (int64_t)a.shape.window + a.shape.sink + a.shape.tok);
  if (rows * (4 * d) * G <= 126 << 20) return 0;
  const int tiles = ChunkSeq{0, a.max_new}.tiles(a.shape.tok);
  int n = 3;
  while (((a.H_kv | G) & ((1 << n) - 1)) || 1 << n > tiles) --n;
  return n;
}

cudaError_t launch_chunk_attend_tc(const ChunkAttendArgs &a, int d, int G, cudaStream_t s) {
  if (a.rows < 256) return launch_chunk_attend_few(a, d, G, s);
  ChunkAttendArgs b = a;
  b.shape.lanes2 = chunk_lanes2(a, d, G);
  return d == 128 ? launch_typed<128>(b, G, s) : launch_typed<64>(b, G, s);
}

}  // namespace lg
