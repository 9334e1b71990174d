// lg_pick_token and lg_count_tokens: from a step's logits to the token on top and its probability.
//
// One pass over a row: each thread keeps the largest processed logit m it has seen, the lowest
// token that has it, and the sum s of exp(x - m) (s falls by exp(m - m') when a larger m' comes),
// and the threads' triples merge in a tree.  A row is split over a cluster of CTAs that merge
// through distributed shared memory, so a batch of one still spreads over 16 SMs.
//
// The penalties touch few tokens: a row's seen bits say which, one bit beside each logit, and the
// count of a token is read only where its bit is set.  Biased tokens get a bit in shared memory;
// only they look through the row's list.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lg_common.cuh"
#include "lg_internal.h"

namespace lg {
namespace {

constexpr int kPickThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Top {
  float m, s;
  int id;
};

// e^(x - m) with x <= m; 1 where they are equal, infinite ones included
__device__ __forceinline__ float share(float x, float m) {
  return x == m ? 1.f : exp2_fast((x - m) * kLog2e);
}

__device__ __forceinline__ Top merge(const Top &a, const Top &b) {
  const bool first = a.m > b.m || (a.m == b.m && a.id <= b.id);
  const Top &w = first ? a : b, &l = first ? b : a;
  Top r = w;
  if (l.m != -INFINITY) r.s += l.s * share(l.m, w.m);
  return r;
}

struct PickArgs {
  const void *x;
  void *out;
  const uint32_t *seen, *allowed;
  const int32_t *counts, *bias_off, *bias_id;
  const float *bias_val;
  const float4 *penalty;
  int32_t *tokens;
  float *pmax;
  int32_t *status;
  int64_t stride;
  int V, words, slice;  // slice: tokens a CTA of the cluster takes, a multiple of 32
};

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// bits t .. t + n - 1 of a row of words (n <= 16, t + n within the row's 32 * words bits)
__device__ __forceinline__ uint32_t bits_at(const uint32_t *w, int t, int words) {
  const int i = t >> 5;
  const uint32_t lo = w[i], hi = i + 1 < words ? w[i + 1] : 0u;
  return __funnelshift_r(lo, hi, t & 31);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}

template <typename T>
__global__ void __launch_bounds__(kPickThreads) pick_token_kernel(PickArgs a, int csize) {
  constexpr int N = 16 / (int)sizeof(T);
  extern __shared__ uint32_t s_biased[];  // [slice / 32] when there are biases
  __shared__ Top s_top[kPickThreads / 32];
  __shared__ Top s_cta;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / csize;
  const int rank = csize > 1 ? (int)cluster_rank() : 0;
  pdl_enter();
  const bool skip = cta_status_bad(a.status);
  Top top{-INFINITY, 0.f, INT_MAX};
  const int lo = rank * a.slice, hi = min(a.V, lo + a.slice);  // this CTA's tokens
  int b0 = 0, b1 = 0;
  if (a.bias_off && !skip) {
    b0 = a.bias_off[b];
    b1 = a.bias_off[b + 1];
    for (int i = tid; i < a.slice / 32; i += kPickThreads) s_biased[i] = 0;
    __syncthreads();
    for (int e = b0 + tid; e < b1; e += kPickThreads) {
      const int t = a.bias_id[e];
      if (t >= lo && t < hi) atomicOr(&s_biased[(t - lo) >> 5], 1u << ((t - lo) & 31));
    }
    __syncthreads();
  }
  if (lo < hi && !skip) {
    const T *x = (const T *)a.x + b * a.stride;
    T *out = a.out ? (T *)a.out + b * a.stride : nullptr;
    const uint32_t *seen = a.seen ? a.seen + (int64_t)b * a.words : nullptr;
    const uint32_t *allowed = a.allowed ? a.allowed + (int64_t)b * a.words : nullptr;
    const int32_t *counts = a.seen ? a.counts + (int64_t)b * a.V : nullptr;
    const float4 pen = a.seen ? a.penalty[b] : make_float4(1.f, 0.f, 0.f, 0.f);
    // one token's processed logit
    auto process = [&](float v, int t, bool was_seen, bool biased, bool ok) {
      if (was_seen) {
        v = v > 0.f ? __fdiv_rn(v, pen.x) : __fmul_rn(v, pen.x);
        const int n = counts[t];
        if (n > 0) v = __fsub_rn(__fsub_rn(v, __fmul_rn(pen.z, (float)n)), pen.y);
      }
      if (biased)
        for (int e = b0; e < b1; ++e)
          if (a.bias_id[e] == t) v = __fadd_rn(v, a.bias_val[e]);
      return ok && v == v ? v : -INFINITY;
    };
    auto add = [&](float v, int t) {
      if (v > top.m) {
        top.s = top.m == -INFINITY ? 0.f : top.s * share(top.m, v);
        top.m = v;
        top.id = t;
      }
      if (v != -INFINITY) top.s += share(v, top.m);
    };
    auto one = [&](int t) {
      const bool s = seen && (seen[t >> 5] >> (t & 31) & 1);
      const bool bi = b0 < b1 && (s_biased[(t - lo) >> 5] >> ((t - lo) & 31) & 1);
      const bool ok = !allowed || (allowed[t >> 5] >> (t & 31) & 1);
      const float v = process(to_float<T>(x[t]), t, s, bi, ok);
      if (out) Elem<T>::store(out, t, v);
      add(v, t);
    };
    // 16-byte vectors where the row is aligned for them, single tokens around
    const int to16 = (int)((16 - ((uintptr_t)(x + lo) & 15)) & 15) / (int)sizeof(T);
    const int v0 = min(hi, lo + to16), nvec = (hi - v0) / N;
    const bool out16 = out && (((uintptr_t)(out + v0)) & 15) == 0;
    if (tid < v0 - lo) one(lo + tid);
    if (tid < hi - v0 - nvec * N) one(v0 + nvec * N + tid);
    const uint4 *xv = (const uint4 *)(x + v0);
    for (int i = tid; i < nvec; i += kPickThreads) {
      const uint4 u = xv[i];
      const int t = v0 + i * N;
      const uint32_t all = (1u << N) - 1;
      const uint32_t sb = seen ? bits_at(seen, t, a.words) & all : 0u;
      const uint32_t ab = allowed ? bits_at(allowed, t, a.words) & all : all;
      const uint32_t bb = b0 < b1 ? bits_at(s_biased, t - lo, a.slice / 32) & all : 0u;
      float f[N];
      Elem<T>::unpack(u, (float2 *)f);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t bit = 1u << e;
        f[e] = process(f[e], t + e, sb & bit, bb & bit, ab & bit);
      }
      if (out) {
        if (out16) {
          uint4 w;
          if constexpr (sizeof(T) == 2) {
            __nv_bfloat162 *h = (__nv_bfloat162 *)&w;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
          } else {
            w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                           __float_as_uint(f[3]));
          }
          *(uint4 *)(out + t) = w;
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) Elem<T>::store(out, t + e, f[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) add(f[e], t + e);
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    Top u;
    u.m = __shfl_xor_sync(0xffffffffu, top.m, o);
    u.s = __shfl_xor_sync(0xffffffffu, top.s, o);
    u.id = __shfl_xor_sync(0xffffffffu, top.id, o);
    // the same order on both sides, so that both get the same bits
    top = (lane & o) ? merge(u, top) : merge(top, u);
  }
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kPickThreads / 32; ++w) top = merge(top, s_top[w]);
    s_cta = top;
  }
  if (csize > 1) {
    cluster_sync();
    if (rank == 0 && tid == 0) {
      const uint32_t mine = smem_addr(&s_cta);
      for (int r = 1; r < csize; ++r) {
        uint32_t at;
        Top u;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(r));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u.m) : "r"(at));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u.s) : "r"(at + 4));
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(u.id) : "r"(at + 8));
        top = merge(top, u);
      }
    }
    cluster_sync();  // the peers' shared memory lives until it has been read
  }
  if (rank == 0 && tid == 0 && !skip) {
    const bool none = top.m == -INFINITY;
    a.tokens[b] = none ? -1 : top.id;
    a.pmax[b] = none ? 0.f : 1.f / top.s;
  }
}

__global__ void count_tokens_kernel(const int32_t *tokens, const int32_t *off, int T, int batch,
                                    int V, int words, int generated, uint32_t *seen,
                                    int32_t *counts, int32_t *status) {
  pdl_enter();
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= T || status_bad(status)) return;
  int b = i;
  if (off) {  // the row that entry i belongs to
    int lo = 0, hi = batch;  // the first bound above i among off[1..batch]
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (off[mid + 1] > i)
        hi = mid;
      else
        lo = mid + 1;
    }
    b = lo;
    if (b >= batch || off[b] > i) return;
  }
  const int t = tokens[i];
  if (t < 0 || t >= V) return;
  atomicOr(&seen[(int64_t)b * words + (t >> 5)], 1u << (t & 31));
  if (generated) atomicAdd(&counts[(int64_t)b * V + t], 1);
}

template <typename T>
cudaError_t launch_pick_typed(PickArgs &a, int batch, cudaStream_t s) {
  // CTAs a row: as many as keep about two CTAs an SM busy, at most 16, each with at least 4096
  // tokens of its own
  int c = 1;
  while (c < 16 && (int64_t)batch * c < 152 && a.V / (2 * c) >= 4096) c *= 2;
  a.slice = ((a.V + c - 1) / c + 31) / 32 * 32;
  const size_t smem = a.bias_off ? (size_t)a.slice / 8 : 0;
  auto kern = pick_token_kernel<T>;
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  if (smem > 32 * 1024)
    LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(batch * c));
  cfg.blockDim = dim3(kPickThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = c;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  LG_TRY(cudaLaunchKernelEx(&cfg, kern, a, c));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pick_token(const lg_logits &x, const uint32_t *seen, const int32_t *counts,
                              const float *penalty, const lg_bias *bias, const uint32_t *allowed,
                              int32_t *tokens, float *pmax, void *logits_out, int32_t *status,
                              cudaStream_t s) {
  PickArgs a = {};
  a.x = x.x;
  a.out = logits_out;
  a.seen = seen;
  a.allowed = allowed;
  a.counts = counts;
  if (bias) a.bias_off = bias->off, a.bias_id = bias->id, a.bias_val = bias->val;
  a.penalty = (const float4 *)penalty;
  a.tokens = tokens;
  a.pmax = pmax;
  a.status = status;
  a.stride = x.stride;
  a.V = x.V;
  a.words = (x.V + 31) / 32;
  return x.dtype == LG_BF16 ? launch_pick_typed<__nv_bfloat16>(a, x.batch, s)
                            : launch_pick_typed<float>(a, x.batch, s);
}

cudaError_t launch_count_tokens(const int32_t *tokens, const int32_t *off, int T, int batch, int V,
                                int generated, uint32_t *seen, int32_t *counts, int32_t *status,
                                cudaStream_t s) {
  if (T == 0) return cudaSuccess;
  LG_TRY(launch_pdl(count_tokens_kernel, (T + 255) / 256, 256, 0, s, tokens, off, T, batch, V,
                    (V + 31) / 32, generated, seen, counts, status));
  return cudaGetLastError();
}

}  // namespace lg
