/*
 * lg_chunk.h -- the model step around the guarded cache: chunks of new tokens (whole prompts,
 * pieces of them, several proposed tokens, or one token a sequence) that join the cache and attend
 * over it, and the token picked from a step's logits.  Part of liblg.so; the conventions of lg.h
 * (caller-owned device memory, asynchronous on the caller's stream, host validation before any
 * launch, the cache's sticky device status) hold for every call here.
 *
 * A prompt, or a chunk of one, on this ABI:
 *   lg_begin_chunk, then for each layer lg_rope_append -> lg_chunk_attend, then lg_pick_token on
 *   the last rows' logits and lg_count_tokens
 * after which the decode steps of lg.h follow.  A decode step whose keys come unrotated is
 * lg_begin_chunk and, for each layer, lg_rope_append -> lg_decode_attend; one whose attention has a
 * sliding window is a chunk of one token a sequence through lg_chunk_attend.
 *
 * What lg_chunk_attend does not do: it returns no statistics (lg_detect cannot follow such a step;
 * lg_token_detect can, from tokens and probabilities) and adds to no H2O scores.  A single token
 * without a window belongs into lg_decode_attend, which does both, in half the time for one short
 * sequence.
 *
 * These calls have no counterpart in the paper (arXiv 2604.10044): its guard reads keys, values,
 * tokens and top-1 probabilities (Sec. 3.1, Sec. 5.2, Eq. 8) that a model step produces here.
 */
#ifndef LG_CHUNK_H
#define LG_CHUNK_H

#include "lg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The new tokens of a batch: row off[b] + j of the token arrays is the j-th new token of sequence
   b, j < m_b = off[b+1] - off[b] (any m_b from 0 to max_new).  Rows outside [off[0], off[batch])
   are neither read into a result nor written. */
typedef struct {
  const int32_t *off; /* device [batch + 1], not falling, off[0] >= 0, off[batch] <= T */
  int32_t T;          /* rows of the token arrays                                      */
  int32_t max_new;    /* host bound on every m_b                                       */
} lg_chunk;

/* Reserves the chunk's slots: len[b] += m_b.  A sequence whose rows would pass cap[b], an m_b
   outside [0, max_new] or an off[] outside [0, T] sets LG_ERR_CAPACITY on the device and leaves
   that sequence's length. */
LG_API lg_status lg_begin_chunk(const lg_cache *c, const lg_chunk *ch, cudaStream_t s);

/* Pairs of a head's first rot elements that are rotated together. */
typedef enum {
  LG_ROPE_HALF = 0,       /* (i, i + rot/2) */
  LG_ROPE_INTERLEAVED = 1 /* (2i, 2i + 1)   */
} lg_rope_layout;

/* How the frequencies f_i = theta^(-2i/rot) are changed for contexts beyond orig_len. */
typedef enum {
  LG_ROPE_PLAIN = 0,  /* f_i                                                               */
  LG_ROPE_LINEAR = 1, /* f_i / factor                                                      */
  LG_ROPE_BASE = 2,   /* theta * factor^(rot/(rot-2)) in place of theta                    */
  LG_ROPE_BANDS = 3,  /* w f_i + (1-w) f_i/factor, w = (orig_len f_i/(2 pi) - low)/(high - low)
                         clamped to [0, 1]: wavelengths over orig_len/low are stretched, those
                         under orig_len/high kept                                          */
  LG_ROPE_YARN = 4    /* w f_i + (1-w) f_i/factor, w = 1 - (i - a)/(b - a) clamped to [0, 1],
                         a and b the (fractional) pair indices that make beta_fast and beta_slow
                         turns over orig_len, rounded down and up and kept in [0, rot-1]; b - a
                         at least 0.001                                                    */
} lg_rope_scaling;

typedef struct {
  int32_t layout;   /* lg_rope_layout                                               */
  int32_t rot;      /* rotated elements of a head: a multiple of 16, 16..d          */
  int32_t scaling;  /* lg_rope_scaling                                              */
  int32_t orig_len; /* BANDS, YARN                                                  */
  double theta;     /* base, > 1                                                    */
  double factor;    /* >= 1; ignored by PLAIN                                       */
  double low, high; /* BANDS, 0 < low < high                                        */
  double beta_fast, beta_slow; /* YARN, beta_fast > beta_slow > 0                   */
  double mscale;    /* factor of the rotated elements (queries and keys), > 0       */
} lg_rope_params;

/* Fills *p: half layout, rot = d, no scaling, orig_len 8192, theta 10000, factor 1, low 1,
   high 4, beta_fast 32, beta_slow 1, mscale 1. */
LG_API lg_status lg_default_rope_params(lg_rope_params *p, int d);

/* Rotary positions of one layer's queries and keys, and the keys and values joining the cache:
   with angle a = pos[t] f_i, a pair (x, y) becomes mscale (x cos a - y sin a, x sin a + y cos a);
   the other elements of a head are copied.  The product with the position is exact modulo a turn;
   the frequency has the 53 bits of a double and some twenty roundings, so an angle is off by less
   than pos[t] f_i 2^-48 radians (1e-6 at position 2^28) beside the fp32 steps after it.
     q_out[t][h][:]                      = rotated q[t][h][:]
     K row len[b] - m_b + j of kv-head h = rotated k_new[t][h][:],  t = off[b] + j
     V row                               = v_new[t][h][:]
   and what lg_append does with a new row: the guard layer's sketch, and on the H2O path the row's
   position (pos[t], required then as everywhere) and a zero score.
   q: device [T][H_q][d] dtype; k_new, v_new: device [T][H_kv][d]; each with its own stride from
   token to token in elements (a multiple of 16 bytes, at least the row), so that slices of one
   projection's output pass as they are.  q_out: device [T][H_q][d] dense; it may be q itself when
   q is dense, and overlaps none of the inputs otherwise.  q and q_out may be null together with
   H_q = 0 (keys and values only).  pos: device [T].  16-byte alignment throughout (pos 4).  Call
   after lg_begin_chunk. */
LG_API lg_status lg_rope_append(const lg_cache *c, const lg_chunk *ch, int layer, const void *q,
                                int64_t q_stride, int H_q, const void *k_new, int64_t k_stride,
                                const void *v_new, int64_t v_stride, const int32_t *pos,
                                const lg_rope_params *rp, void *q_out, const lg_guard_params *p,
                                cudaStream_t s);

/* Workspace bytes lg_chunk_attend needs (partial results of sequences whose rows several CTAs
   share); 0 on invalid arguments.  Over LG_Q4 with more than 64 query rows of a kv-head
   (max_new H_q / H_kv > 64) two more arrays of H_kv S_total d bf16 each, a layer of the whole cache,
   whatever the chunk sees of it: 3.2 times that layer's rows in four bits for d = 128, 2.7 for 64. */
LG_API size_t lg_chunk_workspace_size(const lg_cache *c, const lg_chunk *ch, int H_q, int max_len);

/* Attention of the chunk's queries over the cache (Eq. 1 restricted to what each query may see):
   query j of sequence b belongs to row r = len[b] - m_b + j and sees the rows i <= r; with
   window > 0 only those with i > r - window or i < n_sink (a sliding window and first rows that
   stay visible; window counts the query's own row).
     out[t][h][:] = sum_i a_i v_i,  a = softmax_i(<q[t][h], k_i> * scale) over the rows seen
   q: device [T][H_q][d] dense, dtype; out: device same shape, dtype, may not overlap q.  Query
   head h reads kv-head h / (H_q/H_kv).  What lies in rows that a query does not see never reaches
   its result, whatever it holds.  bf16: the weights enter the product with the values in bf16
   (off by 2^-8 of each at most; lg_decode_attend carries them in two terms over a bf16 cache), scores
   and sums are fp32.  LG_Q4: up to 64 query rows of a kv-head (max_new H_q / H_kv) as lg_decode_attend
   (lg.h); a call with more first writes the rows of every sequence of the chunk that some query sees to
   the workspace as bf16 values, lo + s c rounded, and goes on as over a bf16 cache (3.2e-3 of random
   values' results).  So a sequence's result changes a little, and its time, with the longest chunk that
   shares its call: where one sequence brings a prompt and others a token each, two chunks with a call
   each are better (512 tokens beside 63 single ones, 361000 rows in all: 276 us instead of 566).
   max_len: host bound on every len[b], best a near one, as the division
   of the work (and so the order of sums) goes by it.  A longer sequence sets LG_ERR_CAPACITY, as
   does an m_b above max_new or len[b], or an off[] outside [0, T]; nothing of that call's output is
   then defined.
   ws: device workspace of lg_chunk_workspace_size bytes, 256-byte aligned, any contents; calls
   that may overlap on the GPU need one each. */
LG_API lg_status lg_chunk_attend(const lg_cache *c, const lg_chunk *ch, int layer, const void *q,
                                 int H_q, float scale, int window, int n_sink, void *out,
                                 int max_len, void *ws, size_t ws_bytes, cudaStream_t s);

/* A step's logits: row b is x[b * stride .. b * stride + V). */
typedef struct {
  const void *x;  /* device, dtype                                     */
  int32_t dtype;  /* lg_dtype                                          */
  int32_t batch;  /* rows                                              */
  int32_t V;      /* vocabulary                                        */
  int32_t pad;
  int64_t stride; /* elements from row to row, at least V              */
} lg_logits;

/* Sparse additions to the logits: entries off[b] .. off[b+1] of row b add val[e] to token id[e]
   (entries outside [0, V) are ignored; those of one token add up in the order of e). */
typedef struct {
  const int32_t *off; /* device [batch + 1], not falling, off[0] >= 0 */
  const int32_t *id;  /* device                                       */
  const float *val;   /* device                                       */
} lg_bias;

/* Notes tokens in a batch's history, the state that lg_pick_token's penalties read:
     seen:   device [batch][ceil(V/32)] words, bit j of word w = token 32 w + j has occurred
     counts: device [batch][V] int32, occurrences among the generated tokens
   both zero before a sequence's first tokens.  Tokens of row b: tokens[off[b]] ..
   tokens[off[b+1] - 1], or tokens[b] alone when off is null (a step's picked tokens); T: entries
   of tokens (batch when off is null).  Each sets its seen bit and, when generated, adds one to its
   count (prompt tokens: generated = 0).  Tokens outside [0, V) (a pick of -1) are ignored.
   dev_status: nullable; the call skips its work while it is non-zero. */
LG_API lg_status lg_count_tokens(const int32_t *tokens, const int32_t *off, int T, int batch,
                                 int V, int generated, uint32_t *seen, int32_t *counts,
                                 int32_t *dev_status, cudaStream_t s);

/* The token on top of each row of logits and its probability, after penalties, biases and a
   grammar mask, in fp32 with one rounding an operation:
     seen tokens:      x = x > 0 ? x / repetition : x * repetition
     generated tokens: x = (x - frequency * count) - presence      (count > 0, where seen)
     biases:           x = x + val
     masked tokens:    x = -infinity    (bit clear in allowed; a NaN counts as masked too)
     tokens[b] = the lowest token with the largest x;  pmax[b] = exp(x - max) share of it
   A row with nothing left gives token -1 and pmax 0.  The mass of a row with infinite logits is
   shared evenly among those.
   pmax is of what is left after the penalties, biases and masks: a row with one allowed token has
   pmax 1.  The confidence that lg_token_detect's streak counts is the model's own; where any of the
   three changes the logits, it takes a second call on the logits as they came (seen, bias, allowed
   and logits_out null, other tokens), before this one where this one works in place.  The same call
   again gives the same bits.
   seen, counts: as lg_count_tokens keeps them, both or neither; penalty: device [batch][4]
   {repetition > 0, presence, frequency, unused}, 16-byte aligned, with seen; bias, allowed
   (device [batch][ceil(V/32)] words) nullable.  tokens: device [batch] int32; pmax: device [batch]
   fp32.  logits_out: nullable, device, dtype and stride of x, the processed logits (masked ones
   -infinity) rounded once; may be x itself, or rows that share nothing with x's.  x and logits_out
   need the alignment of their elements only.  dev_status: nullable, a cache's sticky status word. */
LG_API lg_status lg_pick_token(const lg_logits *x, const uint32_t *seen, const int32_t *counts,
                               const float *penalty, const lg_bias *bias, const uint32_t *allowed,
                               int32_t *tokens, float *pmax, void *logits_out,
                               int32_t *dev_status, cudaStream_t s);

#ifdef __cplusplus
}
#endif
#endif
