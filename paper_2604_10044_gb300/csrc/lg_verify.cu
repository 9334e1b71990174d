// Drafted tokens against the target's probabilities, and the rows of those that fall.
//
// lg_verify_draft is two kernels.  The first reads every row of logits once: a CTA a slice of a
// row, kept in registers between its maximum and its sum of exponentials.  The second, a cluster a
// sequence, joins the slices, decides which drafts stand, and looks the random number up in the
// distribution of the one row that the next token comes from.
//
// Which token a number falls on is exact only as far as the sums are: a bound between two tokens
// that moves by 1e-7 of the mass moves past one number in ten million for each of the vocabulary's
// bounds on the way.  So what a lane sums (16 weights) goes into the totals as an integer in units
// of 2^-62 of a mass of one, and integers add up to the same in any order; the quotient by a
// temperature keeps a second term; a row's slices are joined, and its large masses computed, in
// integers too, with powers of two to 2^-38; and a number nearer to a bound than 2^-27 of the mass
// is looked up again with every mass in integers.  Sequences whose token was not the one of 64-bit
// sums: 4 in 10^5 without the large masses and the second search; 4 of 1.44 million so (5 in 10^6
// with a second search from 2^-28 on, 1 in 10^6 from 2^-26 on, met by a third and twice as many calls).
//
// GB300, 261 rows of 128257 bf16 logits of 64 sequences: 19 us in the first kernel (67 MB, 3.5
// TB/s; an element takes some ten instructions, and the CTAs issue in 60 % of the cycles), 21 in
// the second, 40 to 45 a call, 100 or 190 more in the one in ten in which a sequence searches
// twice (100 a round over the row on two SMs): 58 the mean of 60 calls; one sequence's five rows of
// 151936 fp32: 16, of which 13 in the second kernel (the draft's and the slices' loads, two rounds
// over 512 elements a warp, two cluster barriers, all of it latency).  What it took, for 64 sequences
// and for one: loads and work element by element 196 and 59 us; packed fp32 in place of scalar, all
// of a segment loaded first 51 and 21; logits kept packed, lanes' sums in fp32 41 and 20; the
// slices joined in integers instead of in 64-bit floating point 37 and 14; large masses in integers
// 39 and 16; a barrier for the second search 40 and 17.  Not kept: a warp a slice without the CTA's
// barriers 41; two CTAs a sequence more 41 to 50; large weights of the first kernel in integers 49;
// the second search in one CTA 260 to 550 more.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "lg_common.cuh"
#include "lg_internal.h"
#include "lg_rope.cuh"

namespace lg {
namespace {

namespace cg = cooperative_groups;

constexpr int kRowThreads = 256;
constexpr int kRowVecs = 4;  // 16-byte vectors a thread

__host__ __device__ constexpr int slice_elems(int es) { return kRowThreads * kRowVecs * 16 / es; }
// a row that starts inside a vector reaches one vector further
__host__ __device__ inline int row_slices(int V, int es) {
  return (V + 16 / es - 1 + slice_elems(es) - 1) / slice_elems(es);
}

struct RowPart {     // of a slice of a row
  float m;           // largest logit, -infinity where none is left
  int32_t at;        // its lowest place
  uint64_t z;        // sum of exp((x - m) / temperature) in 2^-40
};

// log2(e) / temperature in two terms, the second times ln 2; a temperature of zero (or nothing
// above it) takes the top token.  Temperatures are kept in [2^-60, 2^40] and distances from the
// maximum above -2^60, so every product is a number and what is further down, or masked, weighs
// nothing.
struct Heat {
  float hi, lo;
  bool greedy;
  float lo2;  // the second term as it is
};
constexpr float kFar = -0x1p60f;

__device__ __forceinline__ float clamp_temperature(float t) {
  return t > 0x1p-60f ? fminf(t, 0x1p40f) : 0.f;
}

__device__ __forceinline__ Heat heat_of(float t) {
  Heat h{0.f, 0.f, !(t > 0.f), 0.f};
  if (h.greedy) return h;
  const double e = 1.4426950408889634;
  const float e_hi = (float)e, e_lo = (float)(e - (double)e_hi);
  h.hi = __fdiv_rn(e_hi, t);
  h.lo = __fdiv_rn(__fmaf_rn(-h.hi, t, e_hi) + e_lo, t);
  h.lo2 = h.lo;
  h.lo *= 0.6931471805599453f;
  return h;
}

// exp(d / temperature) of two distances d = x - m from a finite maximum, within some 2^-22 and
// without a drift over the range: 2^y (1 + rest), y the product with the first term
__device__ __forceinline__ float2 weights(float2 d, const Heat &h) {
  d.x = fmaxf(d.x, kFar);
  d.y = fmaxf(d.y, kFar);
  const float2 hi = make_float2(h.hi, h.hi);
  const float2 y = __fmul2_rn(d, hi);
  float2 rest = __ffma2_rn(d, hi, make_float2(-y.x, -y.y));
  rest = __ffma2_rn(rest, make_float2(0.6931471805599453f, 0.6931471805599453f),
                    __fmul2_rn(d, make_float2(h.lo, h.lo)));
  const float2 e = make_float2(exp2_fast(y.x), exp2_fast(y.y));
  return __ffma2_rn(e, rest, e);
}

// v exp((x - m) / temperature), x <= m, in integers (64-bit floating point runs at a hundredth of
// their speed here: it made the joining of slices 5 us of a call), within 2^-38: the exponent is a
// distance without error times two terms, in units of 2^-40; the power of two of its fraction f is
// the series sum of (f ln 2)^k / k!, from k = 5 to 13 in units of 2^-41 in one word, the rest in
// 2^-64 in two.  Out of line: its copies in unrolled loops took longer to fetch than to run.
__device__ __forceinline__ uint64_t scaled_here(uint64_t v, float x, float m, float hi, float lo) {
  if (x == m) return v;
  const float d = x - m, back = d - x, rest = (x - (d - back)) - (m + back);  // x - m = d + rest
  const float y = d * hi;
  if (!(y > -100.f)) return 0;
  const float y2 = __fmaf_rn(d, hi, -y) + __fmaf_rn(d, lo, rest * hi);
  const int64_t e = __float2ll_rn(y * 0x1p40f) + __float2ll_rn(y2 * 0x1p40f);
  const int down = -(int)(e >> 40);
  const uint64_t f = (uint64_t)e << 24;
  const uint32_t g = (uint32_t)(f >> 32);
  uint32_t s = 3u;
  s = 56u + __umulhi(s, g);
  s = 978u + __umulhi(s, g);
  s = 15514u + __umulhi(s, g);
  s = 223818u + __umulhi(s, g);
  s = 2906116u + __umulhi(s, g);
  s = 33541116u + __umulhi(s, g);
  s = 338727216u + __umulhi(s, g);
  s = 2932080444u + __umulhi(s, g);
  uint64_t p = (uint64_t)s << 23;
  p = 177423166116318949ull + __umul64hi(p, f);
  p = 1023870087579328454ull + __umul64hi(p, f);
  p = 4431396893595737425ull + __umul64hi(p, f);
  p = 12786308645202655660ull + __umul64hi(p, f);
  const uint64_t all = v + __umul64hi(v, __umul64hi(p, f));
  return down < 64 ? all >> down : 0;
}
__device__ __noinline__ uint64_t scaled_by(uint64_t v, float x, float m, float hi, float lo) {
  return scaled_here(v, x, m, hi, lo);
}
__device__ __forceinline__ uint64_t scaled(uint64_t v, float x, float m, const Heat &h) {
  return scaled_by(v, x, m, h.hi, h.lo2);
}

template <typename T>
__device__ __forceinline__ float logit(const void *p, int64_t i) {
  const float x = Elem<T>::load(p, i);
  return x == x ? x : -INFINITY;  // a NaN counts as masked
}

// the largest of 16 bytes of logits
template <typename T>
__device__ __forceinline__ float largest(const uint4 &u) {
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162 *h = (const __nv_bfloat162 *)&u;
    const __nv_bfloat162 r = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(r), __high2float(r));
  } else {
    const float *f = (const float *)&u;
    return fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3]));
  }
}

struct VerifyArgs {
  lg_logits x, draft;
  int has_draft, batch, T, max_new, slices;
  const int32_t *off, *tokens;
  const float *temp, *u, *r;
  int32_t *picked, *accepted, *status;
  RowPart *part;  // [T][slices]
};

template <typename T>
__global__ void __launch_bounds__(kRowThreads) verify_rows_kernel(VerifyArgs a) {
  constexpr int kVec = 16 / (int)sizeof(T);
  __shared__ float s_m[kRowThreads / 32];
  __shared__ int s_at[kRowThreads / 32];
  __shared__ uint64_t s_z[kRowThreads / 32];
  __shared__ float s_t;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_enter();
  if (cta_status_bad(a.status)) return;
  const int row = blockIdx.y, V = a.x.V;
  if (warp == 0) {
    const int b = seq_of(a.off, a.batch, row, lane);
    if (lane == 0) s_t = b < 0 ? -1.f : clamp_temperature(a.temp ? a.temp[b] : 1.f);
  }
  const T *x = (const T *)a.x.x + row * a.x.stride;
  const int head = (int)(((uintptr_t)x & 15) / sizeof(T));  // elements of the first vector before the row
  uint4 v[kRowVecs];  // as they are: half the registers for bf16
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k) {
    const int i0 = ((blockIdx.x * kRowVecs + k) * kRowThreads + tid) * kVec - head;
    if (i0 >= 0 && i0 + kVec <= V) {
      v[k] = *(const uint4 *)(x + i0);
    } else {
      T y[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[e] = i0 + e >= 0 && i0 + e < V ? x[i0 + e] : (T)-INFINITY;
      v[k] = *(const uint4 *)y;
    }
  }
  float m = -INFINITY;  // (a maximum passes a NaN over)
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k) m = fmaxf(m, largest<T>(v[k]));
  const float own = m;
  const float wm = warp_max(m);
  if (lane == 0) s_m[warp] = wm;
  __syncthreads();
  const float t = s_t;
  if (t < 0.f) return;  // a row of no sequence
#pragma unroll
  for (int w = 0; w < kRowThreads / 32; ++w) m = fmaxf(m, s_m[w]);
  const Heat h = heat_of(t);
  float2 sums = make_float2(0.f, 0.f);
  int at = 0x7fffffff;
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k) {
    float2 f[kVec / 2];
    Elem<T>::unpack(v[k], f);
    if (m == INFINITY) {
#pragma unroll
      for (int e = 0; e < kVec / 2; ++e) sums.x += (f[e].x == m ? 1.f : 0.f) + (f[e].y == m ? 1.f : 0.f);
    } else if (!h.greedy && m != -INFINITY) {
#pragma unroll
      for (int e = 0; e < kVec / 2; ++e)
        sums = __fadd2_rn(sums, weights(make_float2(f[e].x - m, f[e].y - m), h));
    }
    if (own == m) {
      const int i0 = ((blockIdx.x * kRowVecs + k) * kRowThreads + tid) * kVec - head;
#pragma unroll
      for (int e = 0; e < kVec / 2; ++e) {
        if (f[e].x == m) at = min(at, i0 + 2 * e);
        if (f[e].y == m) at = min(at, i0 + 2 * e + 1);
      }
    }
  }
  uint64_t z = __float2ull_rn((sums.x + sums.y) * 0x1p40f);
#pragma unroll
  for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
  at = __reduce_min_sync(0xffffffffu, at);
  if (lane == 0) {
    s_at[warp] = at;
    s_z[warp] = z;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kRowThreads / 32; ++w) {
      at = min(at, s_at[w]);
      z += s_z[w];
    }
    a.part[(int64_t)row * a.slices + blockIdx.x] = RowPart{m, at, z};
  }
}

// ---------------------------------------------------------------- the decision and the next token

constexpr int kPickThreads = 512;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kSeg = 16;             // elements a lane and segment
constexpr int kSegElems = 32 * kSeg;
constexpr int kSegsKept = ((1 << 20) / kSegElems + kPickWarps - 1) / kPickWarps;  // of a warp, at most
constexpr uint64_t kNear = 1ull << 35;  // in 2^-62: what the fp32 masses are sure of
constexpr int kRowsKept = 64;        // rows of a sequence that are joined once

struct Row {
  float m;    // largest logit
  int at;     // its lowest place
  uint64_t z; // sum of exp((x - m) / temperature) in 2^-40; 0: nothing is left
  float inv_hi, inv_lo;  // 1 / z
  uint64_t inv;          // ... in 2^-63
  int fallen; // the row's draft, -1 for a last row
};

// 1 / z in two terms, and in 2^-63; z in units of 2^-units
__device__ __forceinline__ void reciprocal(Row &r, int units = 40) {
  const float zh = (float)r.z, zl = (float)(int64_t)(r.z - (uint64_t)zh);
  const float inv = __frcp_rn(zh);
  r.inv_hi = inv * __int_as_float((127 + units) << 23);
  r.inv_lo = (__fmaf_rn(-inv, zh, 1.f) - inv * zl) * r.inv_hi;
  r.inv = __float2ull_rn(r.inv_hi * 0x1p62f) * 2 + (uint64_t)__float2ll_rn(r.inv_lo * 0x1p63f);
}

// a row's slices joined; every lane of a warp calls it
__device__ __forceinline__ Row join_row(const VerifyArgs &a, int64_t row, const Heat &h, int lane) {
  const RowPart *p = a.part + row * a.slices;
  Row r{-INFINITY, 0x7fffffff, 0, 0.f, 0.f, 0, -1};
  const RowPart mine = lane < a.slices ? p[lane] : RowPart{-INFINITY, 0, 0};
  r.m = mine.m;
  for (int i = lane + 32; i < a.slices; i += 32) r.m = fmaxf(r.m, p[i].m);
  r.m = warp_max(r.m);
  if (r.m == -INFINITY) return r;
  for (int i = lane; i < a.slices; i += 32) {
    const RowPart s = i == lane ? mine : p[i];
    if (s.m == r.m) r.at = min(r.at, s.at);
    if (!h.greedy && s.z) r.z += scaled(s.z, s.m, r.m, h);
  }
  r.at = __reduce_min_sync(0xffffffffu, r.at);
#pragma unroll
  for (int o = 16; o; o >>= 1) r.z += __shfl_xor_sync(0xffffffffu, r.z, o);
  if (h.greedy) r.z = 1ull << 40;
  if (r.z) reciprocal(r);
  return r;
}

// The draft's probability of a token: what is not above zero (a NaN too) counts as zero.
template <typename Q>
__device__ __forceinline__ float draft_at(const VerifyArgs &a, int64_t row, int i) {
  const float q = Elem<Q>::load((const Q *)a.draft.x + row * a.draft.stride, i);
  return q > 0.f ? q : 0.f;
}

// a mass of [0, 1] in 2^-62, its last bits cut off below 2^-39 (by shifts: the conversion
// instruction for 64 bits took most of this kernel's time)
__device__ __forceinline__ uint64_t units_of(float w) {
  const uint32_t bits = __float_as_uint(w), mant = (bits & 0x7fffffu) | 0x800000u;
  const int sh = (int)(bits >> 23) - (127 - 39);
  return sh >= 0 ? (uint64_t)mant << sh : (uint64_t)(mant >> min(-sh, 31));
}

// rnd of a total, rounded down; the last place for rnd >= 1, the first for what is not above zero
__device__ __forceinline__ uint64_t place_of(float rnd, uint64_t total) {
  if (!(rnd > 0.f) || total == 0) return 0;
  if (rnd >= 1.f) return total - 1;
  const uint32_t bits = __float_as_uint(rnd);  // rnd is mant 2^-(24 + down)
  const uint64_t mant = (bits & 0x7fffffu) | (bits >> 23 ? 0x800000u : 0u);
  const int down = 126 - max((int)(bits >> 23), 1);
  return down < 64 ? __umul64hi(total, mant << 40) >> down : 0;
}

// a lane's elements of a segment, summed in fp32 before they become units (half the work of this
// kernel otherwise): over the lanes of a vocabulary the roundings leave some 2^-30 of the mass
__device__ __forceinline__ uint64_t lane_units(const float (&w)[kSeg]) {
  float2 s = make_float2(w[0], w[1]);
#pragma unroll
  for (int k = 2; k < kSeg; k += 2) s = __fadd2_rn(s, make_float2(w[k], w[k + 1]));
  return units_of(s.x + s.y);
}

struct Part {      // of the vocabulary, a CTA's
  uint64_t total;
  int bad;         // the device status
};

// A CTA of a cluster may send to its peers once they are known to run: each says so on entry, and
// waits for the others before it sends anything, or ends.
__device__ __forceinline__ void peers_arrive() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void peers_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T, typename Q>
__global__ void __launch_bounds__(kPickThreads, 1) verify_pick_kernel(VerifyArgs a) {
  cg::cluster_group cl = cg::this_cluster();
  const int n_cta = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int b = blockIdx.x / n_cta;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ Part s_part[4][16];  // of every CTA of the cluster, for each pass: put there by that CTA
  __shared__ uint64_t s_warp[kPickWarps], s_seg[kPickWarps][kSegsKept];
  __shared__ int s_first, s_bad, s_again;
  __shared__ Row s_row, s_rows[kRowsKept];
  peers_arrive();
  pdl_enter();
  if (tid == 0) s_bad = status_bad(a.status);
  const int o0 = a.off[b], o1 = a.off[b + 1], m = o1 - o0, V = a.x.V;
  const float t = clamp_temperature(a.temp ? a.temp[b] : 1.f);
  const float rnd = a.r[b];
  if (o0 < 0 || m < 0 || m > a.max_new || o1 > a.T) {  // (the same for the cluster)
    if (tid == 0) set_status(a.status, LG_ERR_CAPACITY);
    __syncwarp();
    peers_wait();
    return;
  }
  if (tid == 0) {
    s_first = max(m - 1, 0);
    s_again = 0;
  }
  __syncthreads();
  const Heat h = heat_of(t);
  // a status that is set leaves nothing to do but to meet the cluster's other CTAs, which may have
  // read another one
  const bool bad = s_bad != 0;
  // the first draft that does not stand: a warp a row
  for (int j = warp; j < m && !bad; j += kPickWarps) {
    const int64_t row = o0 + j;
    // (the draft's numbers are asked for before the row's slices)
    const int y = j < m - 1 ? a.tokens[row + 1] : -1;
    const float u = j < m - 1 ? a.u[row] : 0.f;
    float q = 1.f, x = 0.f;
    if (y >= 0 && y < V) {
      if (a.has_draft) q = draft_at<Q>(a, row, y);
      x = logit<T>((const T *)a.x.x + row * a.x.stride, y);
    }
    Row r = join_row(a, row, h, lane);
    if (lane == 0) {
      bool stands = j == m - 1;
      if (y >= 0 && y < V && r.z) {
        // the draft's weight in the same units as z
        const uint64_t e = h.greedy ? (y == r.at ? 1ull << 40 : 0) : scaled(1ull << 62, x, r.m, h);
        stands = u * q * (float)r.z < (float)e * (h.greedy ? 1.f : 0x1p-22f);
      }
      if (!stands) atomicMin(&s_first, j);
      r.fallen = y;
      if (j < kRowsKept) s_rows[j] = r;
    }
  }
  __syncthreads();
  const int first = s_first;
  const int64_t row = o0 + first;
  Row r{-INFINITY, 0x7fffffff, 0, 0.f, 0.f, 0, -1};
  if (m > 0 && !bad) {
    if (first < kRowsKept) {
      r = s_rows[first];
    } else {
      if (warp == 0) {
        Row j = join_row(a, row, h, lane);
        if (lane == 0) {
          j.fallen = first < m - 1 ? a.tokens[row + 1] : -1;
          s_row = j;
        }
      }
      __syncthreads();
      r = s_row;
    }
  }
  const bool fell = first < m - 1;
  const int fallen = r.fallen;
  // the distribution of the next token, p less what the draft had of it
  const T *x = (const T *)a.x.x + row * a.x.stride;
  const Q *dq = a.has_draft && fell && fallen >= 0 && fallen < V
                    ? (const Q *)a.draft.x + row * a.draft.stride
                    : nullptr;
  const float inv_hi = r.inv_hi, inv_lo = r.inv_lo;
  const float far = 0x1p-10f / inv_hi;
  // what is taken off p: nothing, the draft's row, or all of the fallen token
  enum { kNothing, kRow, kToken };
  int less = !fell ? kNothing : dq ? kRow : a.has_draft ? kNothing : kToken;
  // The masses of a lane's elements i0, i0 + step, .. of a segment, but for those (returned as bits)
  // whose share of the row passes 2^-10: their fp32 roundings would not average out.  All loaded first
  // (from the last place on where the row ends: their masses are zeros)
  auto masses_of = [&](auto kind, int i0, int step, float (&w)[kSeg]) -> uint32_t {
    constexpr int kKind = decltype(kind)::value;
    T v[kSeg];
    Q q[kSeg];
    uint32_t big = 0;
#pragma unroll
    for (int k = 0; k < kSeg; ++k) v[k] = x[min(i0 + step * k, V - 1)];
    if constexpr (kKind == kRow) {
#pragma unroll
      for (int k = 0; k < kSeg; ++k) q[k] = dq[min(i0 + step * k, V - 1)];
    }
#pragma unroll
    for (int k = 0; k < kSeg; k += 2) {
      const float va = (float)v[k], vb = (float)v[k + 1];
      float2 e;
      if (r.m == INFINITY) {
        e = make_float2(va == r.m ? 1.f : 0.f, vb == r.m ? 1.f : 0.f);
      } else {  // (a NaN's distance counts as far, like a masked one's)
        e = weights(make_float2(va - r.m, vb - r.m), h);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int i = i0 + step * (k + c);
        const float ec = c ? e.y : e.x;
        float qc = 0.f;
        if constexpr (kKind == kRow) qc = fmaxf((float)q[k + c], 0.f);
        if constexpr (kKind == kToken) qc = i == fallen ? 2.f : 0.f;
        const float p = __fmaf_rn(ec, inv_hi, __fmaf_rn(ec, inv_lo, -qc));
        const bool large = ec > far;
        if (large && i < V) big |= 1u << (k + c);
        w[k + c] = i < V && !large ? fmaxf(p, 0.f) : 0.f;
      }
    }
    return big;
  };
  auto masses = [&](int i0, int step, float (&w)[kSeg]) -> uint32_t {
    if (less == kRow)
      return masses_of(std::integral_constant<int, kRow>(), i0, step, w);
    else if (less == kToken)
      return masses_of(std::integral_constant<int, kToken>(), i0, step, w);
    else
      return masses_of(std::integral_constant<int, kNothing>(), i0, step, w);
  };
  uint64_t inv = r.inv;
  // one mass in integers, in 2^-62, of the weight e in the same units
  auto mass_of = [&](int i, uint64_t e) -> uint64_t {
    const uint64_t p = __umul64hi(e, inv) * 2;
    const float q = less == kRow ? fmaxf((float)dq[i], 0.f) : less == kToken && i == fallen ? 2.f : 0.f;
    const uint64_t off = q < 1.5f ? units_of(q) : ~0ull;
    return p > off ? p - off : 0;
  };
  auto precise = [&](int i) -> uint64_t {
    const float v = (float)x[i];
    return mass_of(i, r.m == INFINITY ? (v == r.m ? 1ull << 62 : 0) : scaled(1ull << 62, v, r.m, h));
  };
  // one times its power of two in line, four at a time: a lane's elements of a segment, summed
  auto all_of = [&](int i0, bool weights_only, int up) -> uint64_t {
    uint64_t sum = 0;
#pragma unroll 4
    for (int k = 0; k < kSeg; ++k) {
      const int i = i0 + 32 * k;
      const float v = i < V ? (float)x[i] : -INFINITY;
      const uint64_t e = r.m == INFINITY ? (v == r.m ? 1ull << up : 0)
                         : v == v        ? scaled_here(1ull << up, v, r.m, h.hi, h.lo2)
                                         : 0;
      if (i < V) sum += weights_only ? e : mass_of(i, e);
    }
    return sum;
  };
  auto warp_sum = [&](uint64_t s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
  };
  // whole segments a warp, in order over the cluster's warps
  const int segs = (V + kSegElems - 1) / kSegElems;
  const int per = (segs + n_cta * kPickWarps - 1) / (n_cta * kPickWarps);
  const int g0 = (rank * kPickWarps + warp) * per, g1 = min(g0 + per, segs);
  const bool look = m > 0 && !bad && !h.greedy && r.z;  // (the top token needs no search)
  uint64_t total = 0, before = 0;
  peers_wait();
  // the sums of the segments and of the warps; of the cluster total, of the CTAs in front before
  auto add_up = [&](int pass, auto segment) -> bool {
    uint64_t s = 0;
    if (look)
      for (int g = g0; g < g1; ++g) {
        const uint64_t sum = warp_sum(segment(g * kSegElems + lane));
        if (lane == 0) s_seg[warp][g - g0] = sum;
        s += sum;
      }
    if (lane == 0) s_warp[warp] = s;
    __syncthreads();
    if (tid < n_cta) {
      uint64_t sum = 0;
#pragma unroll
      for (int w = 0; w < kPickWarps; ++w) sum += s_warp[w];
      cl.map_shared_rank(s_part[pass], tid)[rank] = Part{sum, bad};
    }
    cl.sync();
    total = before = 0;
    bool stop = false;
    for (int c = 0; c < n_cta; ++c) {
      const Part v = s_part[pass][c];
      if (c < rank) before += v.total;
      total += v.total;
      stop |= v.bad != 0;
    }
    return stop;
  };
  for (int pass = 0; pass < 2; ++pass) {  // a second one where the draft leaves nothing: p itself
    const bool stop = add_up(pass, [&](int i0) {
      float w[kSeg];
      uint32_t big = masses(i0, 32, w);
      uint64_t sum = lane_units(w);
      for (; big; big &= big - 1) sum += precise(i0 + 32 * (__ffs(big) - 1));
      return sum;
    });
    if (stop) return;
    if (total || less == kNothing || !look) break;
    less = kNothing;
  }
  // The lowest token whose sum passes r of the total.  Next to a bound between two tokens, nearer
  // than the fp32 masses are sure of, the cluster goes through the row once more, with every mass
  // in integers.
  for (int turn = 0; total; ++turn) {
    const uint64_t want = place_of(rnd, total);
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    if (want >= before && want < before + s_warp[warp]) {  // one warp of the cluster
      int g = g0;
      for (; g < g1 - 1; ++g) {
        const uint64_t sum = s_seg[warp][g - g0];
        if (want < before + sum) break;
        before += sum;
      }
      // the segment again with neighbours in a lane: the lanes' sums, then the elements of one lane.
      // (They may stay short of the sum above by roundings: the last element that has a mass then.)
      const int i0 = g * kSegElems + lane * kSeg;
      uint64_t own = 0, units[kSeg];
      int last = -1;
      uint32_t big = i0 >= V ? 0 : i0 + kSeg <= V ? (1u << kSeg) - 1 : (1u << (V - i0)) - 1;
      if (turn == 0) {
        float w[kSeg];
        big = masses(i0, 1, w);
#pragma unroll
        for (int k = 0; k < kSeg; ++k) units[k] = units_of(w[k]);
      } else {
#pragma unroll
        for (int k = 0; k < kSeg; ++k) units[k] = 0;
      }
      for (; big; big &= big - 1) {
        const int n = __ffs(big) - 1;
        const uint64_t u = precise(i0 + n);
#pragma unroll
        for (int k = 0; k < kSeg; ++k) units[k] = k == n ? u : units[k];
      }
#pragma unroll
      for (int k = 0; k < kSeg; ++k) {
        own += units[k];
        if (units[k]) last = i0 + k;
      }
      uint64_t upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
      }
      const unsigned over = __ballot_sync(0xffffffffu, before + upto > want);
      const unsigned any = __ballot_sync(0xffffffffu, last >= 0);
      // Masses below a unit each leave a segment a sum, of 16 in fp32, but no element: the search in
      // integers settles those, where what an element has is what its segment's sum has of it.
      if (lane == (over ? __ffs((int)over) - 1 : any ? 31 - __clz((int)any) : 0)) {
        uint64_t c = before + upto - own;
        int token = last;
        uint64_t near = 0;  // how far it is to another token
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
          const uint64_t from = c;
          c += units[k];
          if (from <= want && c > want) {
            token = i0 + k;
            // (No token ends where the line begins: r = 0 asks for the first mass.  But next to a draft's
            // row fp32 may leave a mass where there is none, and at the line's end sums of lanes decide.)
            near = min(from == 0 && less != kRow ? UINT64_MAX : want - from, c - 1 - want);
          }
        }
        if (near < kNear && turn == 0)
          for (int c = 0; c < n_cta; ++c) *cl.map_shared_rank(&s_again, c) = 1;
        else
          a.picked[row] = token;
      }
    }
    if (turn) break;
    cl.sync();
    if (!s_again) break;
    if (less == kRow && r.m != INFINITY) {  // (where all masses have one factor it does not count)
      const int up = 38 + __clzll(r.z);     // the sum comes to 2^61 or 2^62
      add_up(2, [&](int i0) { return all_of(i0, true, up); });
      Row sum{r.m, 0, total, 0.f, 0.f, 0, -1};
      reciprocal(sum, up);
      inv = sum.inv;
    }
    add_up(3, [&](int i0) { return all_of(i0, false, 62); });
    if (!total && less != kNothing) {
      less = kNothing;
      add_up(2, [&](int i0) { return all_of(i0, false, 62); });
    }
  }
  if (rank == 0) {
    if (tid == 0) {
      a.accepted[b] = first;
      if (m > 0 && total == 0) a.picked[row] = h.greedy && r.z ? r.at : -1;
    }
    for (int j = tid; j < m; j += kPickThreads)
      if (j != first) a.picked[o0 + j] = j < first ? a.tokens[o0 + j + 1] : -1;
  }
}

// ---------------------------------------------------------------- rows of fallen drafts

__global__ void end_chunk_kernel(lg_cache c, lg_chunk ch, const int32_t *accepted) {
  pdl_enter();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= c.batch) return;
  const int64_t o0 = ch.off[b], o1 = ch.off[b + 1];
  const int n = c.len[b], a = accepted[b];
  if (status_bad(c.dev_status)) return;
  const int64_t m = o1 - o0;
  if (o0 < 0 || m < 0 || o1 > ch.T || m > ch.max_new || m > n || (m > 0 && (a < 0 || a > m - 1)))
    set_status(c.dev_status, LG_ERR_CAPACITY);
  else if (m > 0)
    c.len[b] = n - (int)(m - 1 - a);
}

template <typename T, typename Q>
cudaError_t launch_pick_typed(const VerifyArgs &a, cudaStream_t s) {
  // as many CTAs a sequence as leave each an SM of its own
  int n = 16;
  while (n > 1 && a.batch * n > 152) n /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.batch * n));
  cfg.blockDim = kPickThreads;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (n > 8)
    LG_TRY(cudaFuncSetAttribute(verify_pick_kernel<T, Q>,
                                cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  return cudaLaunchKernelEx(&cfg, verify_pick_kernel<T, Q>, a);
}

template <typename T>
cudaError_t launch_verify_typed(const VerifyArgs &a, cudaStream_t s) {
  if (a.T)  // (a chunk without rows has its counts to set)
    LG_TRY(launch_pdl(verify_rows_kernel<T>, dim3(a.slices, a.T), kRowThreads, 0, s, a));
  return a.draft.dtype == LG_BF16 ? launch_pick_typed<T, __nv_bfloat16>(a, s)
                                  : launch_pick_typed<T, float>(a, s);
}

}  // namespace

size_t verify_ws_bytes(const lg_logits &x, int T) {
  return (size_t)T * row_slices(x.V, x.dtype == LG_BF16 ? 2 : 4) * sizeof(RowPart);
}

cudaError_t launch_verify(const lg_logits &x, const lg_chunk &ch, int batch, const int32_t *tokens,
                          const lg_logits *draft, const float *temp, const float *u, const float *r,
                          int32_t *picked, int32_t *accepted, void *ws, int32_t *status,
                          cudaStream_t s) {
  VerifyArgs a = {};
  a.x = x;
  a.has_draft = draft != nullptr;
  if (draft) a.draft = *draft;
  a.batch = batch, a.T = ch.T, a.max_new = ch.max_new;
  a.slices = row_slices(x.V, x.dtype == LG_BF16 ? 2 : 4);
  a.off = ch.off, a.tokens = tokens;
  a.temp = temp, a.u = u, a.r = r;
  a.picked = picked, a.accepted = accepted, a.status = status;
  a.part = (RowPart *)ws;
  return x.dtype == LG_BF16 ? launch_verify_typed<__nv_bfloat16>(a, s)
                            : launch_verify_typed<float>(a, s);
}

cudaError_t launch_end_chunk(const lg_cache &c, const lg_chunk &ch, const int32_t *accepted,
                             cudaStream_t s) {
  LG_TRY(launch_pdl(end_chunk_kernel, (c.batch + 127) / 128, 128, 0, s, c, ch, accepted));
  return cudaGetLastError();
}

}  // namespace lg
