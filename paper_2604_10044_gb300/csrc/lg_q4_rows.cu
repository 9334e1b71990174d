// Rows of a 4-bit cache: new keys and values rotated, quantised and stored, and rows read back as
// the bf16 values that they stand for.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lg_q4.cuh"
#include "lg_rope.cuh"

namespace lg {
namespace {

// ---------------------------------------------------------------- new rows
//
// A thread holds 16 bytes (8 elements) of a token's heads, one word of codes, or two such where
// halves of the whole head are rotated together.  It takes its cosines and sines once and walks
// over heads: queries (rotated, stored as they are), keys (rotated, rounded to bf16 as a 16-bit
// cache would hold them, quantised), values.  Otherwise the other elements of its pairs come by
// shuffles (so queries may be rotated in place), as do the least and largest element of a group,
// over the 4 (d = 128) or 2 lanes that hold it. (GB300, ragged prompts of up to 4096 tokens, 32
// query heads and 8 of keys and values of 128, 246 MB: 62 us, 4 TB/s, the warps issuing in 64 % of
// the cycles; queries, keys and values in one loop with their pointers chosen a head 95, a word a
// thread with the other half of its pairs by shuffles 103.)

struct Q4AppendArgs {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16 *q_out;
  const int32_t *pos;
  int64_t q_stride, k_stride, v_stride;  // elements from token to token
  int layer, H_q, rot;                   // rot 0: keys come as they are to be held
  int layout;
  float mscale;
  int guard;     // the layer whose V rows are sketched, -1: none
  int groups;    // threads that share a token's heads: every groups-th head each
  int tok;       // tokens a CTA
  int parts;     // CTAs that share a token's heads
  int T;
};

constexpr int kQ4Threads = 256;
constexpr int kQ4Tokens = 64;  // tokens a CTA at most (256 / 4 lanes)
constexpr int kQ4InFlight = 4; // words of a thread in flight

// token_slots in one round trip where a lane can hold a sequence
__device__ __forceinline__ void token_slots_near(const lg_cache &c, const lg_chunk &ch, int t0, int n,
                                                 int64_t *s_slot) {
  const int lane = threadIdx.x & 31;
  if (c.batch < 32) {
    const bool mine = lane < c.batch;
    const int at = lane <= c.batch ? ch.off[lane] : 0x7fffffff;
    const int len = mine ? c.len[lane] : 0, cap = mine ? c.cap[lane] : 0;
    const int64_t seq = mine ? c.seq_off[lane] : 0;
    for (int i = threadIdx.x >> 5; i < n; i += blockDim.x >> 5) {
      const int t = t0 + i;
      const unsigned below = __ballot_sync(0xffffffffu, mine && at <= t);
      const int b = below ? 31 - __clz((int)below) : 0;  // the last sequence that starts at or before t
      const int end = __shfl_sync(0xffffffffu, at, b + 1);
      const int64_t row = (int64_t)__shfl_sync(0xffffffffu, len, b) - end + t;
      const bool in = below && t < ch.T && end > t && row >= 0 && row < __shfl_sync(0xffffffffu, cap, b);
      const int64_t slot = __shfl_sync(0xffffffffu, seq, b) + row;
      if (lane == 0) s_slot[i] = in ? slot : -1;
    }
    return;
  }
  token_slots(c, ch, t0, n, s_slot);
}

// ONE: token t is the one new row of sequence t, and blockIdx.y the layer.  PAIR: halves of the
// whole head are rotated together, so a thread holds both elements of its pairs, words pc and pc +
// D / 16.
template <int D, bool ONE, bool PAIR>
__global__ void __launch_bounds__(kQ4Threads)
    q4_append_kernel(lg_cache c, lg_chunk ch, Q4AppendArgs a, const __grid_constant__ RopeTable tab) {
  constexpr int kW = PAIR ? 2 : 1;  // words of a thread
  constexpr int kTogether = kQ4InFlight / kW;
  constexpr int kLanes = D / 8 / kW, kGroup = D / 32, kRow = q4_row_bytes(D);
  __shared__ int64_t s_slot[kQ4Tokens];
  __shared__ int s_bad;
  // no early trigger: the loop-onset test reads sketches before its own wait
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (threadIdx.x == 0) s_bad = status_bad(c.dev_status);
  const int t0 = blockIdx.x * a.tok;
  const int layer = a.layer + (ONE ? (int)blockIdx.y : 0);
  if constexpr (ONE) {
    for (int i = threadIdx.x; i < a.tok; i += kQ4Threads) {
      const int b = t0 + i;
      int64_t slot = -1;
      if (b < c.batch) {
        const int n = c.len[b];
        const int64_t at = c.seq_off[b];
        if (n > 0) slot = at + n - 1;
        else set_status(c.dev_status, LG_ERR_CAPACITY);
      }
      s_slot[i] = slot;
    }
  } else {
    token_slots_near(c, ch, t0, a.tok, s_slot);
  }
  __syncthreads();
  if (s_bad) return;
  const int pc = threadIdx.x % kLanes;
  const int unit = threadIdx.x / kLanes, i = unit / a.groups;
  const int groups = a.groups * a.parts, grp = blockIdx.z * a.groups + unit % a.groups;
  const int t = t0 + i;
  const int64_t slot = i < a.tok && t < a.T ? s_slot[i] : -1;
  const bool live = slot >= 0;
  // !PAIR: the lane that holds the other elements of the word's pairs
  const bool half_lay = a.layout == LG_ROPE_HALF, turned = PAIR || 8 * pc < a.rot;
  const int hp = a.rot / 16;  // words of half of the rotated elements
  const int other = (threadIdx.x & 31) - pc + (turned && half_lay ? (pc < hp ? pc + hp : pc - hp) : pc);
  float2 co[4], si[4];  // of the elements' pairs; si with the sign of its product with the other element
  if (live && turned && a.rot) {
    const uint64_t p = (uint64_t)(int64_t)a.pos[t];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (PAIR || half_lay) {
        const int pair = (PAIR || pc < hp ? pc : pc - hp) * 8 + 2 * e;
        turn_cos_sin(p * tab.turn[pair], co[e].x, si[e].x);
        turn_cos_sin(p * tab.turn[pair + 1], co[e].y, si[e].y);
        const float m = !PAIR && pc >= hp ? a.mscale : -a.mscale;
        si[e].x *= m;
        si[e].y *= m;
        co[e].y *= a.mscale;
      } else {
        turn_cos_sin(p * tab.turn[pc * 4 + e], co[e].x, si[e].x);
        si[e].x *= -a.mscale;
        si[e].y = -si[e].x;
        co[e].y = co[e].x * a.mscale;
      }
      co[e].x *= a.mscale;
    }
  }
  auto rotated = [&](const uint4 &own, const uint4 &far, bool second) {  // second: of a PAIR
    float2 f[4], g[4];
    Elem<__nv_bfloat16>::unpack(own, f);
    Elem<__nv_bfloat16>::unpack(far, g);
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 o = PAIR || half_lay ? g[e] : make_float2(g[e].y, g[e].x);
      const float2 s = second ? make_float2(-si[e].x, -si[e].y) : si[e];
      const float2 y = __ffma2_rn(f[e], co[e], __fmul2_rn(o, s));
      const __nv_bfloat162 p = __floats2bfloat162_rn(y.x, y.y);
      r[e] = *(const uint32_t *)&p;
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
  };
  const int64_t in = ONE ? (int64_t)blockIdx.y * c.batch + t : t;  // token row of the inputs
  // Heads of one kind, head h of the combined line of queries, keys and values with thread h mod
  // groups. Every lane of a warp makes the same number of turns, as the shuffles need them all; the
  // words of kTogether heads are requested before the first is worked on.
  auto heads = [&](auto kind, const __nv_bfloat16 *src, int before, int count, uint8_t *dst) {
    constexpr int kKind = decltype(kind)::value;  // 0: queries, 1: keys, 2: values
    const int first = (grp - before % groups + groups) % groups;
    const int turns = (count + groups - 1) / groups;
    src += (int64_t)first * D + 8 * pc;
    for (int n0 = 0; n0 < turns; n0 += kTogether) {
      uint4 own[kTogether][kW];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const bool mine = live && first + (n0 + k) * groups < count;
#pragma unroll
        for (int w = 0; w < kW; ++w)
          own[k][w] = mine ? *(const uint4 *)(src + (int64_t)(n0 + k) * groups * D + w * (D / 2))
                           : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        if (n0 + k >= turns) break;
        const int h = first + (n0 + k) * groups;
        const bool mine = live && h < count;
        uint4(&x)[kW] = own[k];
        if (kKind < 2 && a.rot) {
          if constexpr (PAIR) {
            const uint4 y = rotated(x[0], x[1], false);
            x[1] = rotated(x[1], x[0], true);
            x[0] = y;
          } else {
            uint4 far = x[0];
            if (half_lay) {
              far.x = __shfl_sync(0xffffffffu, far.x, other);
              far.y = __shfl_sync(0xffffffffu, far.y, other);
              far.z = __shfl_sync(0xffffffffu, far.z, other);
              far.w = __shfl_sync(0xffffffffu, far.w, other);
            }
            if (turned) x[0] = rotated(x[0], far, false);
          }
        }
        if constexpr (kKind == 0) {
          if (!mine) continue;
#pragma unroll
          for (int w = 0; w < kW; ++w)
            *(uint4 *)(dst + ((int64_t)h * D + 8 * pc + w * (D / 2)) * 2) = x[w];
        } else {
          uint32_t *row = (uint32_t *)(dst + ((int64_t)h * c.S_total + slot) * kRow);
#pragma unroll
          for (int w = 0; w < kW; ++w) {
            float y[8];
            Elem<__nv_bfloat16>::unpack(x[w], (float2 *)y);
            uint32_t par;
            const uint32_t word = q4_encode<kGroup>(y, par);
            if (!mine) continue;
            const int at = pc + w * kLanes;
            row[at] = word;
            if (pc % kGroup == 0) row[D / 8 + at / kGroup] = par;
            if (kKind == 2 && layer == a.guard)  // signs of the values as they came
              ((uint8_t *)c.sketch)[slot * (c.H_kv * D / 8) + h * (D / 8) + at] =
                  (uint8_t)Elem<__nv_bfloat16>::signs(x[w]);
          }
        }
      }
    }
  };
  const int64_t layer_row = (int64_t)layer * c.H_kv * c.S_total * kRow;
  if (a.H_q)
    heads(std::integral_constant<int, 0>(), a.q + in * a.q_stride, 0, a.H_q,
          (uint8_t *)(a.q_out + (int64_t)t * a.H_q * D));
  heads(std::integral_constant<int, 1>(), a.k + in * a.k_stride, a.H_q, c.H_kv,
        (uint8_t *)c.k + layer_row);
  heads(std::integral_constant<int, 2>(), a.v + in * a.v_stride, a.H_q + c.H_kv, c.H_kv,
        (uint8_t *)c.v + layer_row);
}

template <int D, bool ONE, bool PAIR>
cudaError_t launch_append_as(const lg_cache &c, const lg_chunk &ch, Q4AppendArgs &a, int n_layers,
                             const RopeTable &tab, cudaStream_t s) {
  constexpr int kLanes = D / 8 / (PAIR ? 2 : 1);
  const int heads = a.H_q + 2 * c.H_kv;
  // as many heads a thread, for its cosines and sines to serve, as leave the GPU some waves of CTAs
  // (ragged prompts of up to 4096 tokens: one wave 84 us, two 77, four 75, eight 104); a few
  // tokens' heads over several CTAs
  const int64_t full = (int64_t)16 * 152 * kQ4Threads;
  a.groups = 1;
  while (a.groups * 2 <= kQ4Threads / kLanes && a.groups < heads &&
         (int64_t)a.T * n_layers * a.groups * kLanes < full)
    a.groups *= 2;
  a.tok = kQ4Threads / kLanes / a.groups;
  const int64_t ctas = (int64_t)((a.T + a.tok - 1) / a.tok) * n_layers;
  a.parts = 1;
  while (a.parts * a.groups < heads && ctas * a.parts < 2 * 152) a.parts *= 2;
  const dim3 grid((a.T + a.tok - 1) / a.tok, n_layers, a.parts);
  LG_TRY(launch_pdl(q4_append_kernel<D, ONE, PAIR>, grid, kQ4Threads, 0, s, c, ch, a, tab));
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_append_d(const lg_cache &c, const lg_chunk *ch, Q4AppendArgs &a, int n_layers,
                            const RopeTable &tab, cudaStream_t s) {
  const bool pair = a.rot == D && a.layout == LG_ROPE_HALF;
  if (!ch) return launch_append_as<D, true, false>(c, lg_chunk{}, a, n_layers, tab, s);
  return pair ? launch_append_as<D, false, true>(c, *ch, a, n_layers, tab, s)
              : launch_append_as<D, false, false>(c, *ch, a, n_layers, tab, s);
}

// ---------------------------------------------------------------- rows read back

struct Q4ReadArgs {
  int layer;
  __nv_bfloat16 *k_out, *v_out;  // [T][H_kv][d]
  int tok;
};

// the chunk's rows as values: a thread a word, bound by its stores
template <int D>
__global__ void __launch_bounds__(kQ4Threads)
    q4_read_kernel(lg_cache c, lg_chunk ch, Q4ReadArgs a) {
  constexpr int kLanes = D / 8, kGroup = D / 32, kRow = q4_row_bytes(D);
  __shared__ int64_t s_slot[kQ4Tokens];
  __shared__ int s_bad;
  pdl_enter();
  if (threadIdx.x == 0) s_bad = status_bad(c.dev_status);
  const int t0 = blockIdx.x * a.tok;
  token_slots_near(c, ch, t0, a.tok, s_slot);
  __syncthreads();
  if (s_bad) return;
  const int units = c.H_kv * kLanes;
  for (int u = threadIdx.x; u < a.tok * units; u += kQ4Threads) {
    const int i = u / units, x = u - i * units, h = x / kLanes, pc = x % kLanes;
    const int64_t slot = s_slot[i];
    if (slot < 0) continue;
    const int64_t at =
        (((int64_t)a.layer * c.H_kv + h) * c.S_total + slot) * kRow;
    const uint32_t *k = (const uint32_t *)((const uint8_t *)c.k + at);
    const uint32_t *v = (const uint32_t *)((const uint8_t *)c.v + at);
    const int64_t to = ((int64_t)(t0 + i) * c.H_kv + h) * D + 8 * pc;
    const uint32_t kw = k[pc], kp = k[kLanes + pc / kGroup];
    const uint32_t vw = v[pc], vp = v[kLanes + pc / kGroup];
    *(uint4 *)(a.k_out + to) = q4_values(kw, kp);
    *(uint4 *)(a.v_out + to) = q4_values(vw, vp);
  }
}

// A layer's rows as values at the same slots of two 16-bit caches of one layer, for the kernels of
// many query rows: what some query of the chunk sees.  blockIdx = (rows, kv-head, sequence).  Bound
// by its stores: with all loads of a thread's 4 (2) words and parameters of keys and of values
// asked for before the first store 55 us for 8 sequences of 8192 rows (352 MB, 6.4 TB/s), word by
// word 71.
constexpr int kExpandRows = 64;

template <int D>
__global__ void __launch_bounds__(kQ4Threads)
    q4_expand_kernel(lg_cache c, lg_chunk ch, int layer, int window, int sink, __nv_bfloat16 *K,
                     __nv_bfloat16 *V) {
  constexpr int kLanes = D / 8, kGroup = D / 32, kRow = q4_row_bytes(D);
  pdl_enter();
  if (cta_status_bad(c.dev_status)) return;
  const int h = blockIdx.y;
  for (int b = blockIdx.z; b < c.batch; b += gridDim.z) {
    const int n = c.len[b], m = ch.off[b + 1] - ch.off[b];
    if (m <= 0 || n > c.cap[b]) continue;
    const int64_t lo = window ? (int64_t)n - m + 1 - window : 0;  // rows from here on are seen
    for (int64_t r0 = (int64_t)blockIdx.x * kExpandRows; r0 < n;
         r0 += (int64_t)gridDim.x * kExpandRows) {
      if (r0 + kExpandRows <= lo && r0 >= sink) continue;
      const int64_t src = ((int64_t)layer * c.H_kv + h) * c.S_total + c.seq_off[b] + r0;
      const int64_t dst = h * c.S_total + c.seq_off[b] + r0;
      const int rows = n - r0 < kExpandRows ? (int)(n - r0) : kExpandRows;
      if (rows == kExpandRows) {  // all of its loads before the first store
        constexpr int kN = kExpandRows * kLanes / kQ4Threads;
        uint32_t kw[kN], kp[kN], vw[kN], vp[kN];
        const int pc = threadIdx.x % kLanes, i0 = threadIdx.x / kLanes;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          const int64_t at = (src + i0 + n * (kQ4Threads / kLanes)) * kRow;
          const uint32_t *k = (const uint32_t *)((const uint8_t *)c.k + at);
          const uint32_t *v = (const uint32_t *)((const uint8_t *)c.v + at);
          kw[n] = k[pc], kp[n] = k[kLanes + pc / kGroup];
          vw[n] = v[pc], vp[n] = v[kLanes + pc / kGroup];
        }
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          const int64_t to = (dst + i0 + n * (kQ4Threads / kLanes)) * D + 8 * pc;
          *(uint4 *)(K + to) = q4_values(kw[n], kp[n]);
          *(uint4 *)(V + to) = q4_values(vw[n], vp[n]);
        }
        continue;
      }
      for (int u = threadIdx.x; u < rows * kLanes; u += kQ4Threads) {
        const int i = u / kLanes, pc = u % kLanes;
        const uint32_t *k = (const uint32_t *)((const uint8_t *)c.k + (src + i) * kRow);
        const uint32_t *v = (const uint32_t *)((const uint8_t *)c.v + (src + i) * kRow);
        const uint32_t kw = k[pc], kp = k[kLanes + pc / kGroup];
        const uint32_t vw = v[pc], vp = v[kLanes + pc / kGroup];
        *(uint4 *)(K + (dst + i) * D + 8 * pc) = q4_values(kw, kp);
        *(uint4 *)(V + (dst + i) * D + 8 * pc) = q4_values(vw, vp);
      }
    }
  }
}

template <int D>
cudaError_t launch_read_d(const lg_cache &c, const lg_chunk &ch, Q4ReadArgs &a, cudaStream_t s) {
  const int units = c.H_kv * (D / 8);
  a.tok = 2 * kQ4Threads / units;
  a.tok = a.tok < 1 ? 1 : a.tok > kQ4Tokens ? kQ4Tokens : a.tok;
  LG_TRY(launch_pdl(q4_read_kernel<D>, (ch.T + a.tok - 1) / a.tok, kQ4Threads, 0, s, c, ch, a));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_q4_append(const lg_cache &c, int layer0, int n_layers, const void *k_new,
                             const void *v_new, int guard_layer, cudaStream_t s) {
  Q4AppendArgs a = {};
  a.k = (const __nv_bfloat16 *)k_new;
  a.v = (const __nv_bfloat16 *)v_new;
  a.k_stride = a.v_stride = (int64_t)c.H_kv * c.d;
  a.layer = layer0;
  a.guard = c.sketch ? guard_layer : -1;
  a.T = c.batch;
  const RopeTable tab = {};
  return c.d == 128 ? launch_append_d<128>(c, nullptr, a, n_layers, tab, s)
                    : launch_append_d<64>(c, nullptr, a, n_layers, tab, s);
}

cudaError_t launch_q4_rope_append(const lg_cache &c, const lg_chunk &ch, int layer, const void *q,
                                  int64_t q_stride, int H_q, const void *k, int64_t k_stride,
                                  const void *v, int64_t v_stride, const int32_t *pos,
                                  const lg_rope_params &rp, const uint64_t *turns, void *q_out,
                                  bool guard, cudaStream_t s) {
  Q4AppendArgs a = {};
  a.q = (const __nv_bfloat16 *)q;
  a.k = (const __nv_bfloat16 *)k;
  a.v = (const __nv_bfloat16 *)v;
  a.q_out = (__nv_bfloat16 *)q_out;
  a.pos = pos;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.layer = layer, a.H_q = H_q, a.rot = rp.rot, a.layout = rp.layout;
  a.mscale = (float)rp.mscale;
  a.guard = guard ? layer : -1;
  a.T = ch.T;
  RopeTable tab = {};
  for (int i = 0; i < rp.rot / 2; ++i) tab.turn[i] = turns[i];
  return c.d == 128 ? launch_append_d<128>(c, &ch, a, 1, tab, s)
                    : launch_append_d<64>(c, &ch, a, 1, tab, s);
}

cudaError_t launch_q4_read(const lg_cache &c, const lg_chunk &ch, int layer, void *k_out,
                           void *v_out, cudaStream_t s) {
  Q4ReadArgs a = {layer, (__nv_bfloat16 *)k_out, (__nv_bfloat16 *)v_out, 0};
  return c.d == 128 ? launch_read_d<128>(c, ch, a, s) : launch_read_d<64>(c, ch, a, s);
}

cudaError_t launch_q4_expand(const lg_cache &c, const lg_chunk &ch, int layer, int window, int sink,
                             int max_len, void *K, void *V, cudaStream_t s) {
  int gx = (max_len + kExpandRows - 1) / kExpandRows;
  if (gx > 4096) gx = 4096;
  const dim3 grid(gx, c.H_kv, c.batch < 65535 ? c.batch : 65535);
  __nv_bfloat16 *k = (__nv_bfloat16 *)K, *v = (__nv_bfloat16 *)V;
  if (c.d == 128)
    LG_TRY(launch_pdl(q4_expand_kernel<128>, grid, kQ4Threads, 0, s, c, ch, layer, window, sink, k, v));
  else
    LG_TRY(launch_pdl(q4_expand_kernel<64>, grid, kQ4Threads, 0, s, c, ch, layer, window, sink, k, v));
  return cudaGetLastError();
}

}  // namespace lg
