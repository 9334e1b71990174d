// What the kernels that append rotated rows share: the sequence of a token, cache slots, and the
// cosine and sine of an angle given as a fraction of a turn.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "lg_common.cuh"
#include "lg_internal.h"

namespace lg {

struct RopeTable {
  uint64_t turn[64];  // pair i: f_i / 2 pi, in 2^-64 turns
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

}  // namespace lg
