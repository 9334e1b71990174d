// A chunk of new tokens joins the cache: slot reservation, and rotary positions fused with the
// append.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lg_common.cuh"
#include "lg_internal.h"

namespace lg {
namespace {

__global__ void begin_chunk_kernel(lg_cache c, lg_chunk ch) {
  pdl_enter();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= c.batch) return;
  const int64_t o0 = ch.off[b], o1 = ch.off[b + 1];
  const int n = c.len[b], cap = c.cap[b];
  if (status_bad(c.dev_status)) return;
  if (o0 < 0 || o1 < o0 || o1 > ch.T || o1 - o0 > ch.max_new || n + (o1 - o0) > cap)
    set_status(c.dev_status, LG_ERR_CAPACITY);
  else
    c.len[b] = n + (int)(o1 - o0);
}

// ---------------------------------------------------------------- rotary positions and append
//
// The angle of pair i at position p is p f_i radians.  Its size does not matter, only its place in
// the turn, so the frequencies are kept as fractions of a turn in units of 2^-64: p times that,
// modulo 2^64, is the place in the turn, with nothing lost at any 32-bit p, in a few integer
// multiplications.  (In fp32 radians an angle of 10^5 is known to 0.004 only; fp64 would cost 64
// cycles a multiplication and warp here.)  The nearest quarter turn is taken off as an integer
// before the conversion to fp32, so sine and cosine are of at most an eighth of a turn.
//
// A thread owns two 16-byte chunks of a token's heads: for the half layout the chunks that hold
// its pairs' first and second elements, for the interleaved one two chunks of whole pairs.  It
// takes its sines and cosines once and walks over heads.  Queries, then keys; the
// unrotated chunks of a head and the values are copied by the other blocks.

struct RopeTable {
  uint64_t turn[64];  // pair i: f_i / 2 pi, in 2^-64 turns
};

struct RopeArgs {
  const void *q, *k, *v;
  void *q_out;
  const int32_t *pos;
  int64_t q_stride, k_stride, v_stride;  // elements from token to token
  int layer, H_q, rot;
  float mscale;
  int guard;        // the layer's V rows are sketched
  int tok;          // tokens a CTA (rotation)
  int groups;       // threads that share a token's heads: every groups-th head each
  int units;        // threads a token (rotation) = groups * rot chunks / 2
  int rot_blocks;   // CTAs of the rotation part
  int copy_units;   // 16-byte chunks a token in the copy part, whole warps
  int copy_tok;
};

// the sequence that token t belongs to, or -1: 32 bounds at a time, every lane of the warp calls it
__device__ __forceinline__ int seq_of(const int32_t *off, int batch, int t, int lane) {
  int lo = 0, n = batch;  // the answer is in [lo, lo + n); n == 0: none
  // off[lo] <= t must hold for the answer; step through 32 equal parts
  while (true) {
    const int step = (n + 31) / 32;
    const int b = lo + lane * step;
    const bool below = b < lo + n && off[b] <= t;
    const unsigned mask = __ballot_sync(0xffffffffu, below);
    if (mask == 0) return -1;
    const int part = 31 - __clz((int)mask);
    const int end = lo + n;
    lo += part * step;
    n = min(step, end - lo);
    if (step == 1) break;
  }
  return off[lo + 1] > t ? lo : -1;  // the last sequence that starts at or before t (not an empty one)
}

// cache slot (seq_off + row) of each of the CTA's tokens, -1 for none, into s_slot
__device__ __forceinline__ void token_slots(const lg_cache &c, const lg_chunk &ch, int t0, int n,
                                            int64_t *s_slot) {
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < n; i += blockDim.x >> 5) {
    const int t = t0 + i;
    int64_t slot = -1;
    if (t < ch.T) {
      const int b = seq_of(ch.off, c.batch, t, lane);
      if (b >= 0) {
        const int64_t row = (int64_t)c.len[b] - ch.off[b + 1] + t;
        if (row >= 0 && row < c.cap[b]) slot = c.seq_off[b] + row;
      }
    }
    if (lane == 0) s_slot[i] = slot;
  }
}

template <typename T>
__device__ __forceinline__ void store16(T *p, const float *f) {
  uint4 u;
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 *h = (__nv_bfloat162 *)&u;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  } else {
    u = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                   __float_as_uint(f[3]));
  }
  *(uint4 *)p = u;
}

// cosine and sine of the angle `turn` * 2^-64 turns
__device__ __forceinline__ void turn_cos_sin(uint64_t turn, float &co, float &si) {
  const uint32_t hi = (uint32_t)(turn >> 32);
  const uint32_t quad = (hi + 0x20000000u) >> 30;          // nearest quarter turn
  const int32_t rest = (int32_t)(hi - (quad << 30));       // [-1/8, 1/8) turn in 2^-32
  float s, c;
  sincospif((float)rest * 0x1p-31f, &s, &c);
  const float a = (quad & 1) ? s : c, b = (quad & 1) ? c : s;
  co = (quad == 1 || quad == 2) ? -a : a;
  si = (quad & 2) ? -b : b;
}

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 64;  // tokens a CTA at most
constexpr int kTogether = 2;     // heads of a thread in flight

template <typename T, int D>
__global__ void __launch_bounds__(kRopeThreads)
    rope_append_kernel(lg_cache c, lg_chunk ch, RopeArgs a, const __grid_constant__ RopeTable tab,
                       int layout) {
  constexpr int N = 16 / (int)sizeof(T);
  __shared__ int64_t s_slot[kRopeTokens];
  // no early trigger: the loop-onset test reads the sketches before its own wait and re-checks the
  // newest row alone, so a kernel that may write others has to be complete before it starts
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (cta_status_bad(c.dev_status)) return;
  const int64_t row0 = (int64_t)a.layer * c.H_kv * c.S_total;
  T *K = (T *)c.k, *V = (T *)c.v;
  if ((int)blockIdx.x < a.rot_blocks) {
    const int t0 = blockIdx.x * a.tok;
    token_slots(c, ch, t0, a.tok, s_slot);
    __syncthreads();
    const int half = a.rot / 2, pieces = half / N;  // thread's chunk pair
    for (int u = threadIdx.x; u < a.tok * a.units; u += kRopeThreads) {
      const int i = u / a.units, x = u % a.units;
      const int64_t slot = s_slot[i];
      if (slot < 0) continue;
      const int t = t0 + i, grp = x / pieces, pc = x % pieces;
      const int64_t p = a.pos[t];
      float co[N], si[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // half: pair pc N + e; interleaved: N/2 pairs of chunk pc, N/2 of chunk pc + pieces
        const int pair = layout == LG_ROPE_HALF
                             ? pc * N + e
                             : (e < N / 2 ? pc * (N / 2) + e : (pc + pieces) * (N / 2) + e - N / 2);
        turn_cos_sin((uint64_t)p * tab.turn[pair], co[e], si[e]);
        co[e] *= a.mscale;
        si[e] *= a.mscale;
      }
      const int h1 = a.H_q + c.H_kv;
      // kTogether heads' chunks are requested before the first is rotated
      const T *qs = (const T *)a.q + t * a.q_stride + pc * N;
      const T *ks = (const T *)a.k + t * a.k_stride + pc * N;
      T *qd = (T *)a.q_out + (int64_t)t * a.H_q * D + pc * N;
      T *kd = K + (row0 + slot) * D + pc * N;
      for (int h0 = grp; h0 < h1; h0 += kTogether * a.groups) {
        uint4 u0[kTogether], u1[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
          const int h = h0 + k * a.groups;
          if (h >= h1) break;
          const T *src = h < a.H_q ? qs + (int64_t)h * D : ks + (int64_t)(h - a.H_q) * D;
          u0[k] = *(const uint4 *)src;
          u1[k] = *(const uint4 *)(src + half);
        }
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
          const int h = h0 + k * a.groups;
          if (h >= h1) break;
          T *dst = h < a.H_q ? qd + (int64_t)h * D : kd + (h - a.H_q) * c.S_total * D;
          float2 p[N / 2], q[N / 2], y0[N / 2], y1[N / 2];
          Elem<T>::unpack(u0[k], p);
          Elem<T>::unpack(u1[k], q);
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            if (layout == LG_ROPE_HALF) {  // two pairs at a time
              const float2 cc = make_float2(co[2 * e], co[2 * e + 1]);
              const float2 ss = make_float2(si[2 * e], si[2 * e + 1]);
              const float2 neg = make_float2(-ss.x, -ss.y);
              y0[e] = __ffma2_rn(p[e], cc, __fmul2_rn(q[e], neg));
              y1[e] = __ffma2_rn(q[e], cc, __fmul2_rn(p[e], ss));
            } else {  // the pair (x, y): (x, y) c + (-y, x) s
              const int f = e + N / 2;
              y0[e] = __ffma2_rn(p[e], make_float2(co[e], co[e]),
                                 __fmul2_rn(make_float2(-p[e].y, p[e].x), make_float2(si[e], si[e])));
              y1[e] = __ffma2_rn(q[e], make_float2(co[f], co[f]),
                                 __fmul2_rn(make_float2(-q[e].y, q[e].x), make_float2(si[f], si[f])));
            }
          }
          store16<T>(dst, (const float *)y0);
          store16<T>(dst + half, (const float *)y1);
        }
      }
    }
    return;
  }
  // copies: a token's value chunks first (whole warps of consecutive chunks), then the unrotated
  // chunks of its queries and keys, then one unit a kv-head for the row's position and score
  const int t0 = (blockIdx.x - a.rot_blocks) * a.copy_tok;
  token_slots(c, ch, t0, a.copy_tok, s_slot);
  __syncthreads();
  constexpr int kCpr = D / N;
  const int v_units = c.H_kv * kCpr;
  const int plain = (D - a.rot) / N;
  const int qk_units = (a.H_q + c.H_kv) * plain;
  for (int u = threadIdx.x; u < a.copy_tok * a.copy_units; u += kRopeThreads) {
    const int i = u / a.copy_units, x = u % a.copy_units;
    const int64_t slot = s_slot[i];
    if (slot < 0) continue;  // one answer a warp: copy_units is a multiple of 32
    const int t = t0 + i;
    const bool is_v = x < v_units;
    uint4 val = make_uint4(0, 0, 0, 0);
    if (is_v) {
      const int h = x / kCpr, ck = x % kCpr;
      val = *(const uint4 *)((const T *)a.v + t * a.v_stride + (int64_t)x * N);
      *(uint4 *)(V + (row0 + h * c.S_total + slot) * D + ck * N) = val;
    } else if (x < v_units + qk_units) {
      const int y = x - v_units, h = y / plain, e = a.rot + y % plain * N;
      const bool isq = h < a.H_q;
      const T *src = isq ? (const T *)a.q + t * a.q_stride + (int64_t)h * D
                         : (const T *)a.k + t * a.k_stride + (int64_t)(h - a.H_q) * D;
      T *dst = isq ? (T *)a.q_out + ((int64_t)t * a.H_q + h) * D
                   : K + (row0 + (h - a.H_q) * c.S_total + slot) * D;
      if (src != dst) *(uint4 *)(dst + e) = *(const uint4 *)(src + e);
    } else if (c.pos && x < v_units + qk_units + c.H_kv) {
      const int64_t at = row0 + (x - v_units - qk_units) * c.S_total + slot;
      c.pos[at] = a.pos[t];
      c.h2o[at] = 0.f;
    }
    if (a.guard) {  // a word's 32 sign bits from 32 / N neighbouring lanes
      uint32_t w = is_v ? Elem<T>::signs(val) << ((x * N) & 31) : 0u;
#pragma unroll
      for (int o = 1; o < 32 / N; o <<= 1) w |= __shfl_xor_sync(0xffffffffu, w, o);
      if (is_v && (x * N & 31) == 0) c.sketch[slot * (c.H_kv * D / 32) + x * N / 32] = w;
    }
  }
}

template <typename T, int D>
cudaError_t launch_rope_typed(const lg_cache &c, const lg_chunk &ch, RopeArgs &a, int layout,
                              const RopeTable &tab, cudaStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  const int pieces = a.rot / 2 / N, heads = a.H_q + c.H_kv;
  // a warp's threads side by side on one token's heads, so that it reads and writes whole stretches;
  // then as many heads a thread, for its sines and cosines to serve, as leave the GPU four CTAs an SM
  const int64_t full = (int64_t)4 * 152 * kRopeThreads;
  a.groups = pieces < 32 ? 32 / pieces : 1;
  while (a.groups < heads && (int64_t)ch.T * a.groups * pieces < full) a.groups *= 2;
  a.groups = a.groups < heads ? a.groups : heads;
  a.units = a.groups * pieces;
  a.tok = kRopeThreads / a.units;
  a.tok = a.tok < 1 ? 1 : a.tok > kRopeTokens ? kRopeTokens : a.tok;
  a.rot_blocks = (ch.T + a.tok - 1) / a.tok;
  a.copy_units = c.H_kv * (D / N) + heads * ((D - a.rot) / N) + (c.pos ? c.H_kv : 0);
  a.copy_units = (a.copy_units + 31) / 32 * 32;
  a.copy_tok = kRopeThreads * (ch.T * (int64_t)a.copy_units > 4 * full ? 4 : 1) / a.copy_units;
  a.copy_tok = a.copy_tok < 1 ? 1 : a.copy_tok > kRopeTokens ? kRopeTokens : a.copy_tok;
  const int64_t grid = (int64_t)a.rot_blocks + (ch.T + a.copy_tok - 1) / a.copy_tok;
  LG_TRY(launch_pdl(rope_append_kernel<T, D>, dim3((unsigned)grid), kRopeThreads, 0, s, c, ch, a,
                    tab, layout));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_begin_chunk(const lg_cache &c, const lg_chunk &ch, cudaStream_t s) {
  LG_TRY(launch_pdl(begin_chunk_kernel, (c.batch + 127) / 128, 128, 0, s, c, ch));
  return cudaGetLastError();
}

cudaError_t launch_rope_append(const lg_cache &c, const lg_chunk &ch, int layer, const void *q,
                               int64_t q_stride, int H_q, const void *k, int64_t k_stride,
                               const void *v, int64_t v_stride, const int32_t *pos,
                               const lg_rope_params &rp, const uint64_t *turns, void *q_out,
                               bool guard, cudaStream_t s) {
  RopeArgs a = {};
  a.q = q, a.k = k, a.v = v, a.q_out = q_out, a.pos = pos;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.layer = layer, a.H_q = H_q, a.rot = rp.rot;
  a.mscale = (float)rp.mscale;
  a.guard = guard ? 1 : 0;
  RopeTable tab = {};
  for (int i = 0; i < rp.rot / 2; ++i) tab.turn[i] = turns[i];
  if (c.dtype == LG_BF16)
    return c.d == 128 ? launch_rope_typed<__nv_bfloat16, 128>(c, ch, a, rp.layout, tab, s)
                      : launch_rope_typed<__nv_bfloat16, 64>(c, ch, a, rp.layout, tab, s);
  return c.d == 128 ? launch_rope_typed<float, 128>(c, ch, a, rp.layout, tab, s)
                    : launch_rope_typed<float, 64>(c, ch, a, rp.layout, tab, s);
}

}  // namespace lg
