// Rows of a 4-bit cache (lg.h, LG_Q4) and what the kernels that read and write them share.
//
// A head of d elements is four groups of d / 4.  Its row is d / 8 words of eight codes, element 2i
// of a word in bits 4i and element 2i + 1 in bits 16 + 4i, i < 4, so that one shift and one mask
// leave a pair of neighbours in the halves of a word; then a word a group, bf16 scale s below bf16
// least value lo.  A code c stands for lo + s c.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lg_common.cuh"
#include "lg_internal.h"
#include "lg_q4_plan.cuh"

namespace lg {

__host__ __device__ constexpr int q4_row_bytes(int d) { return d / 2 + 16; }

// A group whose range reaches this, or that holds a NaN or an infinity, is held as NaN: weights of
// up to 2^8 times a scale stay within fp32 and bf16.
constexpr float kQ4Range = 0x1p118f;
constexpr uint32_t kQ4NaN = 0x7fffu;  // the word of such a group: scale NaN, least value 0

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Masked codes of a word as they stand: c (bits 0-3 of either half) or 16 c (bits 4-7) in units of
// 2^-133, the least bf16 number.
constexpr uint32_t kQ4Low = 0x000f000fu, kQ4High = 0x00f000f0u;

// the eight values of a word as bf16, lo + s c rounded once: a code times 2^127 is c / 64 or c / 4
// exactly, which 64 s or 4 s make up for
__device__ __forceinline__ uint4 q4_values(uint32_t word, uint32_t par) {
  auto two = [](uint32_t x) { return *(const __nv_bfloat162 *)&x; };
  const __nv_bfloat162 by = two(0x7f007f00u);
  const __nv_bfloat162 s = two(__byte_perm(par, par, 0x1010));
  const __nv_bfloat162 lo = two(__byte_perm(par, par, 0x3232));
  const __nv_bfloat162 s64 = __hmul2(s, two(0x42804280u)), s4 = __hmul2(s, two(0x40804080u));
  auto value = [&](uint32_t raw, const __nv_bfloat162 &scale) {
    const __nv_bfloat162 r = __hfma2(__hmul2(two(raw), by), scale, lo);
    return *(const uint32_t *)&r;
  };
  const uint32_t up = word >> 8;
  return make_uint4(value(word & kQ4Low, s64), value(word & kQ4High, s4), value(up & kQ4Low, s64),
                    value(up & kQ4High, s4));
}

// The word of eight elements and their group's parameter word.  LANES neighbouring lanes hold the
// group; every lane of the warp calls it.
//
// A code is the integer nearest to (x - lo) / s, ties to even.  The product with 1 / s is within
// 2^-22 of the quotient, which settles all but quotients next to a half: with s of 8 bits and a
// code of 4 the residual x - lo - s c is exact, and where none of the eight is half a step or more
// from its code the codes are right.  Otherwise the quotients are divided out (s (c + 1/2) has 13
// bits, so a correctly rounded quotient of 24-bit numbers is never a half that it should not be).
template <int LANES>
__device__ __forceinline__ uint32_t q4_encode(const float *x, uint32_t &par) {
  float lo = x[0], hi = x[0], odd = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
    odd = __fmaf_rn(x[e], 0.f, odd);  // NaN where an element is not finite
  }
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    odd += __shfl_xor_sync(0xffffffffu, odd, o);
  }
  const float range = hi - lo;  // lo is one of the elements, so a bf16 number
  const __nv_bfloat16 sb = __float2bfloat16_rn(range * (1.f / 15.f));
  float s = __bfloat162float(sb);
  if (!(range < kQ4Range) || odd != 0.f) {  // (an odd that is NaN differs from zero)
    par = kQ4NaN;
    return 0;
  }
  if (s < 0x1p-126f) s = 0.f;  // a range that has no normal scale: every element is held as lo
  par = (__float_as_uint(s) >> 16) | (__float_as_uint(lo) & 0xffff0000u);
  if (s == 0.f) return 0;
  const float inv = __frcp_rn(s), half = 0.5f * s;
  constexpr float kRound = 12582912.f;  // 1.5 2^23: the sum's low bits are the nearest integer
  float c[8], worst = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float d = x[e] - lo;
    c[e] = __fmaf_rn(d, inv, kRound);
    worst = fmaxf(worst, fabsf(__fmaf_rn(kRound - c[e], s, d)));
  }
  if (worst >= half) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = kRound + fminf(rintf(__fdiv_rn(x[e] - lo, s)), 15.f);
  }
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) w |= (__float_as_uint(c[e]) & 15u) << (4 * (e / 2) + 16 * (e % 2));
  return w;
}

// D = A B + C, bf16 operands: m16 n8 k16
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                         float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// attention of few query rows over a 4-bit cache (lg_q4_attend.cu)
struct Q4AttendArgs {
  const uint8_t *K, *V;    // cache rows
  const void *q;           // [n_layers][T][H_q][d] bf16
  void *out;               // the same
  float *stats;            // nullable [n_layers][batch][H_q][4] (one new token a sequence)
  const int64_t *seq_off;
  const int32_t *len;
  const int32_t *off;      // nullable [batch + 1]; null: one token a sequence
  int32_t *status;
  float *part;             // [n_layers][ctas][2][rows][d + 4]
  int64_t S_total;
  int layer0, n_layers, batch, H_kv, g, T, max_new, max_len;
  int ctas;                // of a layer
  int cluster;             // CTAs of an item that joins its results itself; 0: items in a line
  int suffix_w;
  float qscale;            // softmax scale * log2(e)
  Q4Shape shape;
};

// how a call is divided, and the bytes of its partial results
struct Q4Grid {
  int rows, ctas, cluster;
  size_t part_bytes;
};
Q4Grid q4_grid(int n_layers, int batch, int H_kv, int g, int d, int max_new, int max_len, int window,
               int sink);
cudaError_t launch_q4_attend(const Q4AttendArgs &a, int d, cudaStream_t s);

// the kernels' grids fit their limits
inline bool q4_grid_fits(int n_layers, int batch, int H_kv) {
  return n_layers <= 65535 && batch <= 65535 && H_kv <= 1 << 20;
}

// the arguments that both calls fill alike
inline void q4_fill(Q4AttendArgs &a, const lg_cache &c, int g, float scale, const Q4Grid &grid,
                    void *ws) {
  a.K = (const uint8_t *)c.k;
  a.V = (const uint8_t *)c.v;
  a.seq_off = c.seq_off;
  a.len = c.len;
  a.status = c.dev_status;
  a.part = (float *)ws;
  a.S_total = c.S_total;
  a.batch = c.batch;
  a.H_kv = a.shape.H_kv = c.H_kv;
  a.g = a.shape.g = g;
  a.shape.rows = grid.rows;
  a.ctas = grid.ctas;
  a.cluster = grid.cluster;
  a.qscale = scale * 1.4426950408889634f;
}

// Query rows of a kv-head above which a call expands the layer's rows to bf16 for the kernels of
// 16-bit caches.  (us, the codes themselves and expanded, 4 query heads of 128, 16 sequences of
// 8192 rows: 32 query rows 103 and 209, 64 178 and 215, 96 257 and 215; 32 sequences of 1000: 48
// and 62, 74 and 71, 101 and 73.)
constexpr int kQ4FewRows = 64;

}  // namespace lg
