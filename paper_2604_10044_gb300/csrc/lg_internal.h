// Internal launch interfaces between the C ABI (lg_api.cu) and the kernel files.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "lg.h"
#include "lg_chunk.h"
#include "lg_draft.h"

namespace lg {

// argument checks shared by the calls (lg_api.cu)
lg_status check_cache(const lg_cache *c);
lg_status check_params(const lg_guard_params *p);

struct AttendArgs {
  const void *K, *V;       // cache [L][H_kv][S_total][d]
  const void *q;           // [n_layers][batch][H_q][d]
  const int64_t *seq_off;  // [batch]
  const int32_t *len;      // [batch]
  int32_t *status;
  float *partial;          // [n_layers][batch][H_q][max_chunks][d + 8]
  float *logits;           // nullable [n_layers][H_kv][S_total][g], log2 units
  int *counter;            // [1 + n_layers * batch * H_kv], zeroed by each call (bf16 pass):
                           // the chunk counter, then chunks done per (layer, sequence, kv-head)
  void *out;               // [n_layers][batch][H_q][d] dtype
  float *stats;            // [n_layers][batch][H_q][4]
  float *final_ml;         // nullable [n_layers][batch][H_q][2]: merged (M, l), log2 units
  int64_t S_total;
  int layer0, n_layers, batch, H_kv, H_q;
  int chunk_rows;          // rows per CTA, a multiple of the tile
  int max_chunks;
  int max_len;
  int suffix_w;
  float qscale;            // softmax scale * log2(e)
  int *gate;               // nullable, else `counter`: both passes are launched, and the cluster
                           // pass leaves -1 in its first word when it has done the call, or clears
                           // the counters for the general pass after it
  int sms;                 // of the GPU (cluster pass)
};

int attend_tile_rows(int dtype, int d);
cudaError_t launch_attend(const AttendArgs &a, int dtype, int d, int g, int64_t rows_total,
                          void *out, float *stats, float *final_ml, float *h2o, cudaStream_t s);
// tensor-core partial pass for bf16 caches (lg_attend_mma.cu)
int mma_tile_rows();
cudaError_t launch_attend_mma_partial(const AttendArgs &a, int d, int g, int64_t rows_total,
                                      cudaStream_t s);

// the cluster pass (lg_attend_cluster.cuh): whether it can take a call, and the call (*general set:
// the general pass is to be launched, instead or, with a.gate set, after it)
bool attend_cluster_takes(const AttendArgs &a, int tile_rows, int64_t rows_total);
cudaError_t launch_attend_cluster(AttendArgs &a, int d, int g, int64_t rows_total,
                                  bool *general, cudaStream_t s);
int cluster_f32_tile_rows();
cudaError_t launch_attend_cluster_f32(AttendArgs &a, int d, int g, int64_t rows_total,
                                      bool *general, cudaStream_t s);

// guard kernels (lg_guard.cu)
cudaError_t launch_begin_step(const lg_cache &c, cudaStream_t s);
cudaError_t launch_append(const lg_cache &c, int layer0, int n_layers, const void *k_new,
                          const void *v_new, const int32_t *pos_new, int guard_layer,
                          cudaStream_t s);
cudaError_t launch_sketch_build(const lg_cache &c, int guard_layer, int max_len, cudaStream_t s);
cudaError_t launch_state_init(const lg_cache &c, lg_guard_state *state, int t_gen0,
                              cudaStream_t s);
// kept_idx nullable: when set, the retained set is formed in the same kernel (no compaction)
cudaError_t launch_detect(const lg_cache &c, const float *stats, int H_q, lg_guard_state *state,
                          const int32_t *budget, const lg_guard_params &p, int32_t *flags,
                          int32_t *spans, double *diag, void *dstate, int32_t *kept_idx,
                          int32_t *kept_count, int max_keep, int max_len, cudaStream_t s);
size_t detect_state_bytes(const lg_cache &c, const lg_guard_params &p);
int detect_smem_rows(const lg_guard_params &p);
size_t detect_smem_bytes(const lg_guard_params &p, int nwords);
cudaError_t launch_prune_compact(const lg_cache &c, const int32_t *flags, const int32_t *spans,
                                 const lg_guard_state *state, const int32_t *budget,
                                 const lg_guard_params &p, int32_t *kept_idx,
                                 int32_t *kept_count, int max_keep, int max_len, cudaStream_t s);
cudaError_t launch_compact(const lg_cache &c, const int32_t *kept_idx, const int32_t *kept_count,
                           int max_keep, cudaStream_t s);
// token-level monitor (lg_token.cu)
size_t token_state_words(const lg_guard_params &p, const lg_token_params &tp);
size_t token_smem_bytes(const lg_guard_params &p, const lg_token_params &tp);
// budget non-null: the kernel also writes this step's kept lists over kept_idx/kept_count
cudaError_t launch_token_detect(const lg_cache &c, const int32_t *tokens, const float *pmax,
                                int32_t *kept_idx, int32_t *kept_count, int max_keep,
                                lg_guard_state *state, const lg_guard_params &p,
                                const lg_token_params &tp, int32_t *flags, int32_t *spans,
                                double *diag, void *tstate, const int32_t *budget, int max_len,
                                cudaStream_t s);
cudaError_t launch_h2o_reset(const lg_cache &c, int max_len, cudaStream_t s);
cudaError_t launch_h2o_evict(const lg_cache &c, const int32_t *budget, const int32_t *pos_now,
                             int max_len, cudaStream_t s);
cudaError_t launch_streaming_evict(const lg_cache &c, const int32_t *budget,
                                   const int32_t *pos_now, int n_sink, int max_len,
                                   cudaStream_t s);


// chunks of new tokens (lg_chunk.cu)
cudaError_t launch_begin_chunk(const lg_cache &c, const lg_chunk &ch, cudaStream_t s);
// turns: rp.rot / 2 frequencies in 2^-64 turns; guard: the layer's V rows are sketched
cudaError_t launch_rope_append(const lg_cache &c, const lg_chunk &ch, int layer, const void *q,
                               int64_t q_stride, int H_q, const void *k, int64_t k_stride,
                               const void *v, int64_t v_stride, const int32_t *pos,
                               const lg_rope_params &rp, const uint64_t *turns, void *q_out,
                               bool guard, cudaStream_t s);

// rows of a 4-bit cache (lg_q4_rows.cu): new ones, one or a chunk a sequence, and read back; expand:
// layer's rows that some query of the chunk sees, at the same slots of one bf16 layer
cudaError_t launch_q4_append(const lg_cache &c, int layer0, int n_layers, const void *k_new,
                             const void *v_new, int guard_layer, cudaStream_t s);
cudaError_t launch_q4_rope_append(const lg_cache &c, const lg_chunk &ch, int layer, const void *q,
                                  int64_t q_stride, int H_q, const void *k, int64_t k_stride,
                                  const void *v, int64_t v_stride, const int32_t *pos,
                                  const lg_rope_params &rp, const uint64_t *turns, void *q_out,
                                  bool guard, cudaStream_t s);
cudaError_t launch_q4_read(const lg_cache &c, const lg_chunk &ch, int layer, void *k_out,
                           void *v_out, cudaStream_t s);
cudaError_t launch_q4_expand(const lg_cache &c, const lg_chunk &ch, int layer, int window, int sink,
                             int max_len, void *K, void *V, cudaStream_t s);

// drafted tokens (lg_verify.cu)
size_t verify_ws_bytes(const lg_logits &x, int T);
cudaError_t launch_verify(const lg_logits &x, const lg_chunk &ch, int batch, const int32_t *tokens,
                          const lg_logits *draft, const float *temp, const float *u, const float *r,
                          int32_t *picked, int32_t *accepted, void *ws, int32_t *status,
                          cudaStream_t s);
cudaError_t launch_end_chunk(const lg_cache &c, const lg_chunk &ch, const int32_t *accepted,
                             cudaStream_t s);

// lg_chunk_attend (lg_chunk_attend.cu): the grid and tiles of a call, and the call
struct ChunkGrid {
  int ctas;  // of the persistent kernel
  int rows;  // of an item
  int tok;   // tokens of an item
  int bn2;   // log2 of the rows of a key block
};
struct ChunkAttendArgs;
ChunkGrid chunk_grid(int dtype, int d, int g, int max_new);
cudaError_t launch_chunk_attend(ChunkAttendArgs &a, int dtype, int d, int G, cudaStream_t s);

// picked tokens (lg_pick.cu)
cudaError_t launch_pick_token(const lg_logits &x, const uint32_t *seen, const int32_t *counts,
                              const float *penalty, const lg_bias *bias, const uint32_t *allowed,
                              int32_t *tokens, float *pmax, void *logits_out, int32_t *status,
                              cudaStream_t s);
cudaError_t launch_count_tokens(const int32_t *tokens, const int32_t *off, int T, int batch, int V,
                                int generated, uint32_t *seen, int32_t *counts, int32_t *status,
                                cudaStream_t s);

}  // namespace lg
