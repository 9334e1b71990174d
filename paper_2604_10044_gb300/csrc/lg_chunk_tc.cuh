// What the two tensor-core kernels of lg_chunk_attend share: waits, the queue of pieces, which blocks
// hide rows, and clearing what is not a number from such blocks.
#pragma once
#include <cuda_bf16.h>

#include "lg_chunk_attend.cuh"
#include "lg_tcgen05.cuh"

namespace lg {

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// bit e: the query at row qrow sees row i0 + e, e < 32
// (hid: the last row that the window hides from it, -1 for none)
__device__ __forceinline__ uint32_t rows_seen(const ChunkShape &s, int qrow, int hid, int i0) {
  auto below = [](int n) {  // bits 0 .. n - 1; shifts of 32 and more give 0
    uint32_t r;
    asm("shr.b32 %0, %1, %2;" : "=r"(r) : "r"(0xffffffffu), "r"(max(32 - n, 0)));
    return r;
  };
  return below(qrow + 1 - i0) & (~below(hid + 1 - i0) | below(s.sink - i0));
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

// the same for a converged warp: one answer, known to be the same in every lane
template <typename B>
__device__ __forceinline__ bool tc_wait_warp(B &b, uint64_t *bar, uint32_t parity) {
  return __all_sync(0xffffffffu, tc_wait(b, bar, parity));
}

// a value that is the same in every lane, as the compiler can know it
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// an element of a bf16 pair that is infinite or NaN: bit 15 or 31 of the result
__device__ __forceinline__ uint32_t not_numbers(uint32_t w) {
  return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// Clears a value block from row i0 of a sequence of n rows, `nthreads` threads together; whether
// something of the sequence's own rows was cleared (by this thread).
template <int BYTES, int BN>
__device__ __forceinline__ bool clear_block(uint8_t *block, int i0, int n, int t, int nthreads) {
  uint4 *v = (uint4 *)block;
  bool bad = false;
  for (int e = t; e < BYTES / 16; e += nthreads) {
    uint4 u = v[e];
    uint32_t *uw = (uint32_t *)&u;
    if (not_numbers(u.x) | not_numbers(u.y) | not_numbers(u.z) | not_numbers(u.w)) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t b = not_numbers(uw[x]);
        uw[x] &= (b & 0x8000u ? 0u : 0xffffu) | (b & 0x80000000u ? 0u : 0xffff0000u);
      }
      v[e] = u;
      bad |= i0 + e / 8 % BN < n;
    }
  }
  return bad;
}

// A piece of work as the roles of a CTA read it.  The copying thread walks along the CTA's share
// (64-bit arithmetic that every role would otherwise repeat, in registers that the rows' warps need
// for scores) and queues the pieces in shared memory, kPieces of them at most.
struct TcPiece {
  TileRows rows;
  TileBlocks blocks;
  int blk0, blk1;         // key blocks; blk1 < 0: no more pieces
  int open0, open1;       // of them, the last run that hides no row: [open0, open1)
  int n;                  // rows of the sequence
  int tok0, tokens, kvh;  // token rows [tok0, tok0 + tokens), kv-head
  int slot;               // of the partial result, -1: the piece is its whole item
  volatile int bad;       // something that is not a number was cleared
  int64_t row0;           // first cache row

  __device__ __forceinline__ bool hides(int blk) const { return blk < open0 || blk >= open1; }
};
constexpr int kPieces = 4;

struct TcQueue {
  uint64_t full[kPieces], empty[kPieces];
  TcPiece piece[kPieces];

  __device__ __forceinline__ void init(int readers) {
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], readers);
    }
  }
  // piece i into its slot; false when a wait ran out
  template <typename B, typename W>
  __device__ __forceinline__ bool put(B &b, uint32_t i, const W &w, const ChunkAttendArgs &a) {
    if (!tc_wait(b, &empty[i % kPieces], ((i / kPieces) & 1) ^ 1)) return false;
    TcPiece &p = piece[i % kPieces];
    p.rows = w.rows;
    p.blocks = w.blocks;
    p.blk0 = w.blk0;
    p.blk1 = w.blk1;
    open_blocks(w.rows, a.shape, w.blocks, p.open0, p.open1);
    p.n = w.q.n;
    p.tok0 = w.off + w.t * a.shape.tok;
    p.tokens = w.tokens(a);
    p.kvh = w.kvh;
    p.slot = w.whole() ? -1 : w.slot();
    p.bad = 0;
    p.row0 = w.row0;
    mbar_arrive(&full[i % kPieces]);
    return true;
  }
  template <typename B>
  __device__ __forceinline__ void end(B &b, uint32_t i) {
    if (!tc_wait(b, &empty[i % kPieces], ((i / kPieces) & 1) ^ 1)) return;
    piece[i % kPieces].blk1 = -1;
    mbar_arrive(&full[i % kPieces]);
  }
  template <typename B>
  __device__ __forceinline__ bool wait(B &b, uint32_t i) {  // whole warp
    return tc_wait_warp(b, &full[i % kPieces], (i / kPieces) & 1);
  }
  __device__ __forceinline__ TcPiece &at(uint32_t i) { return piece[i % kPieces]; }
  __device__ __forceinline__ void done(uint32_t i) { mbar_arrive(&empty[i % kPieces]); }
};

// the queries [T][H_q][d] in boxes of 64 columns, g heads and `tokens` tokens (lg_chunk_attend_tc.cu)
bool make_q_map(CUtensorMap *m, const void *q, int d, int H_q, int T, int g, int tokens);

}  // namespace lg
