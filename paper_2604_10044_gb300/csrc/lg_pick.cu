// lg_pick_token and lg_count_tokens: from a step's logits to the token on top and its probability.
//
// One pass over a row: each thread keeps the largest processed logit m it has seen, the lowest
// token that has it, and the sum s of exp(x - m) (s falls by exp(m - m') when a larger m' comes),
// and the threads' triples merge in a tree.  A row is split over a cluster of CTAs that send theirs
// to the first CTA through distributed shared memory, so a batch of one still spreads over many SMs.
//
// The call reads the logits once and is bound by that, so a thread does little for a vector of 16
// bytes: its maximum, and an exponential an element.  The penalties touch few tokens: a row's seen
// bits say which, one bit beside each logit.  Those tokens, and the biased ones, are listed first and
// left out of the pass; they are processed after it, a thread each, so that the reads of their
// counts wait together.  What is left for the pass is one bit a token in shared memory; a vector
// with no bit set is not even read.  A listed token's place is a prefix sum over the threads' bits, so
// that the same thread adds it to the same sum in every call: pmax is the same bits for the same call.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "lg_common.cuh"
#include "lg_internal.h"

namespace lg {
namespace {

constexpr int kAhead = 4;     // vectors of a thread in flight
constexpr int kAside = 2048;  // listed tokens of a CTA
constexpr float kLog2e = 1.4426950408889634f;

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

// bits sh .. sh + 31 of two words, sh < 32
__device__ __forceinline__ uint32_t window(const uint32_t *w, int sh) {
  return __funnelshift_r(w[0], w[1], sh);
}

// the largest element of 16 bytes, NaN if one is
template <typename T>
__device__ __forceinline__ float max16(const uint4 &u);
template <>
__device__ __forceinline__ float max16<__nv_bfloat16>(const uint4 &u) {
  const __nv_bfloat162 *h = (const __nv_bfloat162 *)&u;
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return __bfloat162float(__hmax_nan(m.x, m.y));
}
template <>
__device__ __forceinline__ float max16<float>(const uint4 &u) {
  auto two = [](float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  };
  const float *f = (const float *)&u;
  return two(two(f[0], f[1]), two(f[2], f[3]));
}

// 16 bytes with the elements whose bit is clear set to -infinity
template <typename T>
__device__ __forceinline__ uint4 keep(const uint4 &u, uint32_t bits) {
  uint4 w = u;
  uint32_t *h = (uint32_t *)&w;
  if constexpr (sizeof(T) == 2) {
    const uint32_t two = (bits & 0x55u) | (bits & 0xaau) << 15;  // a pair's bits 16 apart
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t mask = (two >> (2 * e) & 0x00010001u) * 0xffffu;
      h[e] = (h[e] & mask) | (0xff80ff80u & ~mask);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = bits >> e & 1 ? h[e] : 0xff800000u;
  }
  return w;
}

template <typename T>
__device__ __forceinline__ uint4 pack16(const float *f) {
  if constexpr (sizeof(T) == 2) {
    uint4 w;
    __nv_bfloat162 *h = (__nv_bfloat162 *)&w;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
    return w;
  } else {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
}

// the lanes' triples merged, the same in every lane
__device__ __forceinline__ Top warp_top(const Top &t) {
  Top r;
  r.m = warp_max(t.m);
  r.id = (int)__reduce_min_sync(0xffffffffu, (unsigned)(t.m == r.m ? t.id : INT_MAX));
  r.s = t.m == -INFINITY ? 0.f : t.s * share(t.m, r.m);
#pragma unroll
  for (int o = 16; o; o >>= 1) r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
  return r;
}

constexpr int kMaxCluster = 16;
constexpr int kMinFew = 2 << 10;       // tokens a CTA takes at least: of few rows
constexpr int kMinSlice = 8 << 10;     // of more
constexpr int kMaxSlice = 320 << 10;   // and at most: 16 bytes of bits for every 32
constexpr int kTwoBits = 204 << 10;    // and of two on an SM
constexpr int kFourBits = 88 << 10;    // and of four

template <typename T, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) pick_token_kernel(PickArgs a, int csize) {
  constexpr int N = 16 / (int)sizeof(T);
  constexpr uint32_t kAll = (1u << N) - 1;
  // [4][slice / 32 + 1]: allowed tokens, those of the pass, listed ones, biased ones
  extern __shared__ uint32_t s_bits[];
  __shared__ Top s_top[NT / 32];
  __shared__ float s_max[NT / 32];
  __shared__ Top s_ranks[kMaxCluster];
  __shared__ int s_seen[NT / 32];   // seen tokens of each warp's bits
  __shared__ int s_fit;             // entries of the list that hold one
  __shared__ int s_list[kAside];
  __shared__ int s_twice;           // some token is biased more than once
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / csize, rank = blockIdx.x % csize;
  if (csize > 1)  // (waited for before anything is sent: the peers have started)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  pdl_enter();
  if (tid == 0) {
    s_twice = 0;
    s_fit = kAside;
  }
  const bool skip = cta_status_bad(a.status);
  Top top{-INFINITY, 0.f, INT_MAX};  // of the tokens processed one by one
  float m = -INFINITY, sum = 0.f;    // of this thread's vectors
  int best = 0;                      // the first vector that has m
  const int lo = rank * a.slice, hi = skip ? lo : min(a.V, lo + a.slice);  // this CTA's tokens
  if (lo < hi) {
    const T *x = (const T *)a.x + b * a.stride;
    T *out = a.out ? (T *)a.out + b * a.stride : nullptr;
    const uint32_t *seen = a.seen ? a.seen + (int64_t)b * a.words : nullptr;
    const uint32_t *allowed = a.allowed ? a.allowed + (int64_t)b * a.words : nullptr;
    const int32_t *counts = a.seen ? a.counts + (int64_t)b * a.V : nullptr;
    const float4 pen = a.seen ? a.penalty[b] : make_float4(1.f, 0.f, 0.f, 0.f);
    const int w0 = lo >> 5, nw = ((hi + 31) >> 5) - w0, sw = a.slice / 32 + 1;
    uint32_t *s_ok = s_bits, *s_pass = s_bits + sw, *s_apart = s_bits + 2 * sw,
             *s_bias = s_bits + 3 * sw;
    int b0 = 0, b1 = 0;
    if (a.bias_off) {
      b0 = a.bias_off[b];
      b1 = a.bias_off[b + 1];
    }
    // the penalties of a seen token with its count
    auto penalised = [&](float v, int n) {
      v = v > 0.f ? __fdiv_rn(v, pen.x) : __fmul_rn(v, pen.x);
      return n > 0 ? __fsub_rn(__fsub_rn(v, __fmul_rn(pen.z, (float)n)), pen.y) : v;
    };
    // one more token
    auto add = [&](float v, int t) { top = merge(top, Top{v, v == -INFINITY ? 0.f : 1.f, t}); };
    auto finish = [&](float v, int t) {  // a token processed by itself
      v = v == v ? v : -INFINITY;
      if (out) Elem<T>::store(out, t, v);
      add(v, t);
    };
    // n listed tokens, their logits and counts read together
    auto apart = [&](const int *t, int n) {
      float v[kAhead];
      int c[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        v[k] = k < n ? Elem<T>::load(x, t[k]) : 0.f;
        c[k] = k < n ? counts[t[k]] : 0;
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (k < n) finish(penalised(v[k], c[k]), t[k]);
    };

    // the bits: every token, or the allowed ones, but for the seen and biased ones
#pragma unroll 4
    for (int i = tid; i < nw; i += NT) {
      const int left = a.V - ((w0 + i) << 5);
      const uint32_t ok =
          (allowed ? __ldg(allowed + w0 + i) : ~0u) & (left >= 32 ? ~0u : (1u << left) - 1);
      s_ok[i] = ok;
      s_pass[i] = ok;
      s_apart[i] = seen ? __ldg(seen + w0 + i) & ok : 0u;
      s_bias[i] = 0;
    }
    if (b0 < b1) {
      __syncthreads();
      for (int e = b0 + tid; e < b1; e += NT) {
        const int t = a.bias_id[e] - lo;
        if (t >= 0 && t < hi - lo) {
          const uint32_t bit = s_pass[t >> 5] & 1u << (t & 31);
          if (atomicOr(&s_bias[t >> 5], bit) & bit) s_twice = 1;
        }
      }
      __syncthreads();
    }
    int mine = 0;  // seen tokens of this thread's words, the biased ones aside
    for (int i = tid; i < nw; i += NT) {
      const uint32_t w = s_apart[i] & ~s_bias[i];
      s_pass[i] &= ~(w | s_bias[i]);
      s_apart[i] = w;
      mine += __popc(w);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) s_seen[warp] = mine;
    __syncthreads();

    // 16-byte vectors where the row is aligned for them, single tokens around
    const int to16 = (int)((16 - ((uintptr_t)(x + lo) & 15)) & 15) / (int)sizeof(T);
    const int v0 = min(hi, lo + to16), nvec = (hi - v0) / N;
    const bool out16 = out && (((uintptr_t)(out + v0)) & 15) == 0;
    const uint4 *xv = (const uint4 *)(x + v0);
    // a thread's vectors are NT vectors apart: whole words of bits, at one place in a word
    constexpr int kStep = NT * N / 32;
    const int sh = (v0 - lo + tid * N) & 31;
    const uint32_t *pass0 = s_pass + ((v0 - lo + tid * N) >> 5), *ok0 = pass0 - sw;
    for (int i0 = tid; i0 < nvec; i0 += kAhead * NT, pass0 += kAhead * kStep, ok0 += kAhead * kStep) {
      uint4 u[kAhead];
      uint32_t kb[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * NT;
        kb[k] = 0;
        u[k] = make_uint4(0, 0, 0, 0);
        if (i >= nvec) continue;
        kb[k] = window(pass0 + k * kStep, sh) & kAll;
        if (kb[k] || out) u[k] = __ldcs(xv + i);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * NT, t = v0 + i * N;
        uint4 w = u[k];
        float vm = max16<T>(w), f[N];
        if (vm != vm) {
          Elem<T>::unpack(w, (float2 *)f);
#pragma unroll
          for (int e = 0; e < N; ++e) f[e] = f[e] == f[e] ? f[e] : -INFINITY;
          w = pack16<T>(f);
          vm = max16<T>(w);
        }
        uint32_t left = kAll;  // tokens that w holds still
        if (out && i < nvec) {  // (listed tokens are written again after the pass)
          if (allowed) left = window(ok0 + k * kStep, sh) & kAll;
          if (left != kAll) w = keep<T>(w, left);
          if (out16) {
            __stcs((uint4 *)(out + t), w);
          } else {
            const T *h = (const T *)&w;
#pragma unroll
            for (int e = 0; e < N; ++e) out[t + e] = h[e];
          }
        }
        if (kb[k] != left) w = keep<T>(w, kb[k]);
        if (kb[k] != kAll) vm = max16<T>(w);
        Elem<T>::unpack(w, (float2 *)f);
        best = vm > m ? i : best;
        const float m1 = fmaxf(m, vm), base = m1 == -INFINITY ? 0.f : m1;
        sum *= exp2_fast((m - base) * kLog2e);
        m = m1;
        float2 p[N / 2];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          const float2 d = __fadd2_rn(make_float2(f[2 * e], f[2 * e + 1]), make_float2(-base, -base));
          const float2 z = __fmul2_rn(d, make_float2(kLog2e, kLog2e));
          p[e] = make_float2(exp2_fast(z.x), exp2_fast(z.y));
        }
#pragma unroll
        for (int w = N / 4; w; w /= 2)
#pragma unroll
          for (int e = 0; e < w; ++e) p[e] = __fadd2_rn(p[e], p[e + w]);
        sum += p[0].x + p[0].y;
      }
    }
    // the ends of the row, then the listed tokens
    auto one = [&](int t) {
      if (!(s_pass[(t - lo) >> 5] >> ((t - lo) & 31) & 1)) {
        if (out && allowed && !(allowed[t >> 5] >> (t & 31) & 1)) Elem<T>::store(out, t, -INFINITY);
        return;
      }
      float v = Elem<T>::load(x, t);
      v = v == v ? v : -INFINITY;
      if (out) Elem<T>::store(out, t, v);
      add(v, t);
    };
    if (tid < v0 - lo) one(lo + tid);
    if (tid < hi - v0 - nvec * N) one(v0 + nvec * N + tid);
    const int of = lane < NT / 32 ? s_seen[lane] : 0;
    const int listed = __reduce_add_sync(0xffffffffu, of);
    // The words' tokens into the list, in the order of warps, then of words: neighbouring entries are
    // neighbouring tokens mostly (192 rows 40.2 us; in the order of threads, whose words stand apart,
    // 41.1), and the prefix sums wait until the list is needed (one row 6.9 us; before the pass, with a
    // barrier more, 7.7).
    if (mine) {
      int at = __reduce_add_sync(0xffffffffu, lane < warp ? of : 0);
      auto put = [&](int i, uint32_t w, int at) {
        if (w == 0) return;
        if (at + __popc(w) > kAside) {  // (the word stays, and so does every later one)
          if (at < kAside) s_fit = at;
          return;
        }
        s_apart[i] = 0;
        for (; w; w &= w - 1) s_list[at++] = lo + 32 * i + __ffs((int)w) - 1;
      };
      for (int i = tid; i - lane < nw; i += 2 * NT) {  // two words a lane, their places summed together
        const uint32_t w = i < nw ? s_apart[i] : 0u, w2 = i + NT < nw ? s_apart[i + NT] : 0u;
        const int own = __popc(w) | __popc(w2) << 16;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += u;
        }
        const int all = __shfl_sync(0xffffffffu, sum, 31);
        sum -= own;
        put(i, w, at + (sum & 0xffff));
        at += all & 0xffff;
        put(i + NT, w2, at + (sum >> 16));
        at += all >> 16;
      }
    }
    __syncthreads();  // (and the pass has stored their logits as they came)
    if (__builtin_expect(listed > kAside, 0))
      for (int i = tid; i < nw; i += NT)
        for (uint32_t w = s_apart[i]; w; w &= w - 1) {
          const int t[kAhead] = {lo + 32 * i + __ffs((int)w) - 1};
          apart(t, 1);
        }
    const int n = min(listed, s_fit);
    for (int i = tid; i < n; i += kAhead * NT) {
      int t[kAhead], k1 = 0;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        t[k] = 0;
        if (i + k * NT < n) {
          t[k] = s_list[i + k * NT];
          k1 = k + 1;
        }
      }
      apart(t, k1);
    }
    // biased tokens, each by the thread of its first entry
    for (int e = b0 + tid; e < b1; e += NT) {
      const int t = a.bias_id[e];
      if (t < lo || t >= hi) continue;
      if (!(s_bias[(t - lo) >> 5] >> ((t - lo) & 31) & 1)) continue;  // (masked)
      if (__builtin_expect(s_twice, 0)) {
        int f = b0;
        while (a.bias_id[f] != t) ++f;
        if (f < e) continue;
      }
      float v = Elem<T>::load(x, t);
      if (seen && (seen[t >> 5] >> (t & 31) & 1)) v = penalised(v, counts[t]);
      if (__builtin_expect(s_twice, 0)) {
        for (int f = e; f < b1; ++f)
          if (a.bias_id[f] == t) v = __fadd_rn(v, a.bias_val[f]);
      } else {
        v = __fadd_rn(v, a.bias_val[e]);
      }
      finish(v, t);
    }
    // the CTA's maximum; the token only from threads whose vectors have it
    const float wm = warp_max(fmaxf(m, top.m));
    if (lane == 0) s_max[warp] = wm;
    __syncthreads();
    const float cm = warp_max(s_max[lane & (NT / 32 - 1)]);
    Top vec{m, sum, INT_MAX};
    if (m == cm && cm != -INFINITY) {
      if (cm == INFINITY) vec.s = 0.f;
      for (int i = best; i < nvec; i += NT) {
        const int at = v0 + i * N;
        const uint32_t kb = window(s_pass + ((at - lo) >> 5), (at - lo) & 31) & kAll;
        for (int e = N - 1; e >= 0; --e)
          if ((kb >> e & 1) && Elem<T>::load(x, at + e) == m) {
            vec.id = min(vec.id, at + e);
            if (cm == INFINITY) vec.s += 1.f;
          }
        if (cm != INFINITY) break;
      }
    }
    top = merge(top, vec);
  }
  top = warp_top(top);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  if (warp == 0) top = warp_top(lane < NT / 32 ? s_top[lane] : Top{-INFINITY, 0.f, INT_MAX});
  if (csize > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid == 0) {  // to the first CTA
      uint32_t at;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(&s_ranks[rank])), "r"(0));
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(top.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(top.s) : "memory");
      asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at + 8), "r"(top.id) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::
                     : "memory");
    if (rank == 0 && warp == 0)
      top = warp_top(lane < csize ? s_ranks[lane] : Top{-INFINITY, 0.f, INT_MAX});
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

template <typename T, int NT>
cudaError_t pick_config(cudaLaunchConfig_t &cfg, cudaLaunchAttribute *attr, int batch, int c,
                        size_t smem) {
  auto kern = pick_token_kernel<T, NT>;
  LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  // (every call sets the same limit: another thread's call may come between it and the launch)
  if (smem > 36 * 1024)
    LG_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (kMaxSlice / 32 + 1) * 4 * (int)sizeof(uint32_t)));
  cfg.gridDim = dim3((unsigned)(batch * c));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = smem;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = c;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaSuccess;
}

// Clusters of c CTAs that run at once: a cluster stands within one GPC, so those of more CTAs leave
// some of the GPU's places empty.  Asked once a size and device, for bits that leave an SM all the CTAs
// that it has threads for.  (With the bits of a slice of 208 K tokens and more, one CTA of 512 threads
// fits an SM instead of two; dividing by that instead was slower: 140 rows of 500000 57 -> 67 us.)
constexpr int kDevices = 16;
template <typename T, int NT>
int clusters_at_once(int c) {
  static std::atomic<int> known[kDevices][kMaxCluster + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::atomic<int> *const at = dev < kDevices ? &known[dev][c] : nullptr;
  int n = at ? at->load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    if (pick_config<T, NT>(cfg, attr, 1, c, 32 * 1024) != cudaSuccess) return 0;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, pick_token_kernel<T, NT>, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      n = 0;
    }
    if (at) at->store(n, std::memory_order_relaxed);
  }
  return n;
}

template <typename T, int NT>
cudaError_t launch_pick_typed(PickArgs &a, int batch, int c, cudaStream_t s) {
  a.slice = ((a.V + c - 1) / c + 31) / 32 * 32;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  // (a word more each: a vector's bits are read from two)
  LG_TRY((pick_config<T, NT>(cfg, attr, batch, c,
                             (size_t)(a.slice / 32 + 1) * 4 * sizeof(uint32_t))));
  cfg.stream = s;
  LG_TRY(cudaLaunchKernelEx(&cfg, pick_token_kernel<T, NT>, a, c));
  return cudaGetLastError();
}

// CTAs a row, of 512 threads (two an SM): the most whose clusters run at once, at most ten, each with
// 8192 tokens or more (16, and 2048, where rows are so few that every CTA finds an SM of its own), and
// enough that a slice's bits fit shared memory.  Rows too many for two CTAs each and not for three of
// 256 threads (four an SM) take those, while their bits leave room for two an SM; rows too many for one
// of 512 threads take one of 256, as long as four CTAs' bits fit an SM.  Measured on a GB300, calls
// back to back, us by threads x CTAs a row:
//   rows of 128257 bf16:   8  512x10  6.8, 512x16  8.2     16  512x8  7.8, 512x16 12.5 (do not fit)
//                         48  512x5  11.1, 512x6  16.0    152  512x2 16.1, 256x4  23.2
//                        192  256x3  22.0, 512x1  25.0    256  512x1 25.7, 256x2  26.9
//                        608  512x1  52.6, 256x1  79.3 (three an SM)
//   180 rows of bf16: of 320000 (room for three an SM) 256x3 48, 512x1 62; of 500000 (two) 256x3 69,
//                     512x2 83; of 900000 (one) 256x3 210, 512x3 129
//   rows of 32000 bf16:   16  512x3   6.8, 512x10  7.7    608  256x1 17.2, 512x1  21.4
//   rows of 32000 fp32:    1  512x15  5.6, 512x3   6.6
template <typename T>
cudaError_t launch_pick_sized(PickArgs &a, int batch, cudaStream_t s) {
  const int least = (a.V + kMaxSlice - 1) / kMaxSlice;
  const bool few = batch <= 4;
  int c = few ? kMaxCluster : 10, most = a.V / (few ? kMinFew : kMinSlice);
  c = c > most ? (most < 1 ? 1 : most) : c;
  while (c > 1 && clusters_at_once<T, 512>(c) < batch) --c;
  if (c == 1 && a.V <= 3 * kTwoBits && most >= 3 && batch <= clusters_at_once<T, 256>(3))
    return launch_pick_typed<T, 256>(a, batch, 3, s);
  c = c < least ? least : c;
  if (c == 1 && a.V <= kFourBits && batch > clusters_at_once<T, 512>(1))
    return launch_pick_typed<T, 256>(a, batch, 1, s);
  return launch_pick_typed<T, 512>(a, batch, c, s);
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
  return x.dtype == LG_BF16 ? launch_pick_sized<__nv_bfloat16>(a, x.batch, s)
                            : launch_pick_sized<float>(a, x.batch, s);
}

cudaError_t launch_count_tokens(const int32_t *tokens, const int32_t *off, int T, int batch, int V,
                                int generated, uint32_t *seen, int32_t *counts, int32_t *status,
                                cudaStream_t s) {
  if (T == 0) return cudaSuccess;
  LG_TRY(launch_pdl(count_tokens_kernel, ((unsigned)T + 255) / 256, 256, 0, s, tokens, off, T, batch, V,
                    (V + 31) / 32, generated, seen, counts, status));
  return cudaGetLastError();
}

}  // namespace lg
