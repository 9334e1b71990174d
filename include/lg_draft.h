/*
 * lg_draft.h -- several tokens a step: what drafted tokens of a chunk stand against the target model,
 * the rows of the others leaving the cache, and the rows of a 4-bit cache read back.  Part of liblg.so;
 * the conventions of lg.h hold for every call here.
 *
 * A decode step that checks k drafted tokens a sequence on this ABI: the chunk of a sequence is its last
 * token and its drafts, m_b = k_b + 1 rows (any k_b, none too), and
 *   lg_begin_chunk, for each layer lg_rope_append -> lg_chunk_attend, then
 *   lg_verify_draft on the chunk's logits -> lg_end_chunk -> lg_count_tokens on what was picked
 * after which row 0 of the next chunk is picked[off[b] + accepted[b]].
 * The monitors of lg.h do not follow such a step: lg_chunk_attend gives lg_detect no statistics, and
 * lg_token_detect takes one token a call, whose row is the cache's last, where the rows of all drafts
 * have joined before any is checked.  A guarded decode is one of single tokens.
 *
 * These calls have no counterpart in the paper (arXiv 2604.10044), which decodes a token a step.
 */
#ifndef LG_DRAFT_H
#define LG_DRAFT_H

#include "lg_chunk.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Workspace bytes lg_verify_draft needs (a few numbers a slice of a row); 0 on invalid arguments. */
LG_API size_t lg_verify_workspace_size(const lg_logits *x, const lg_chunk *ch);

/* Which drafted tokens stand, and the token that follows them.  Row t = off[b] + j of x holds the
   target's logits after token tokens[t] of sequence b; for j < m_b - 1 the draft of what follows is
   y = tokens[t + 1].  With temperature tau_b:
     p_t(i) = exp((x_t(i) - max x_t) / tau_b) / sum of the same; for tau_b = 0 (and what is not above
              2^-60, or NaN) one for the lowest token with the largest logit; for tau_b > 2^40 as for
              2^40.  A NaN counts as -infinity; the mass of a row with infinite logits is shared
              evenly among those; a row with nothing left has p = 0
     q_t(i)   the probability that the draft gave i: row t of `draft` (an entry that is not above zero
              counts as zero), or, without `draft`, one for i = y and zero elsewhere
     draft j stands when all before it do and u[t] q_t(y) < p_t(y)
     accepted[b] = the number of drafts that stand, a
     the next token is drawn from row t = off[b] + a with weights w = max(p_t - q_t, 0), or p_t where a
              counts all drafts or the w are all zero (to 2^-60 of the mass): the lowest i with
              sum_{k <= i} w(k) > r[b] sum w.  r below zero or NaN counts as 0, from one on as just
              below one.  -1 where p_t = 0
     picked[off[b] + j] = draft j for j < a, the next token for j = a, -1 for j > a
   so that the tokens of sequence b are distributed as the target's whatever the draft is, when u and r
   are uniform on [0, 1) and independent.  A draft outside [0, V) falls, with q_t = 0.
   A weight is within about 2^-22 (2^-38 from 2^-10 of the mass on); what 16 of them sum to is added up in
   integers, in units of 2^-62 of the mass (2^-40 of the largest weight in p's own sum), so the same call
   gives the same tokens.  Where r falls within 2^-27 of the mass of a bound between two tokens, or of the end of
   the last one, the row is gone through again with every weight within 2^-38: a call with such a sequence takes
   100 to 200 us more.  (r = 0, the start of the first, is as good as any other number, but next to p - q, for
   which the row is gone through again there too.)
   x: rows [0, T) at least (x->batch >= T); draft: nullable, as many rows of the same V, its own dtype and
   stride.  tokens: device [T]; temperature: nullable (1), device [batch]; u: device [T] (the entry of a
   sequence's last row is not used); r: device [batch]; picked: device [T], accepted: device [batch];
   they overlap nothing else.  Rows outside [off[0], off[batch]) are not touched.  m_b = 0: accepted[b] = 0.
   V up to 2^20, T up to 65535.  ws: device, lg_verify_workspace_size bytes, 16-byte aligned, any
   contents; calls that may overlap on the GPU need one each.  dev_status: nullable, a cache's sticky
   status word: the call skips its work while it is non-zero, and an m_b outside [0, max_new] or an
   off[] outside [0, T] sets LG_ERR_CAPACITY. */
LG_API lg_status lg_verify_draft(const lg_logits *x, const lg_chunk *ch, int batch,
                                 const int32_t *tokens, const lg_logits *draft,
                                 const float *temperature, const float *u, const float *r,
                                 int32_t *picked, int32_t *accepted, void *ws, size_t ws_bytes,
                                 int32_t *dev_status, cudaStream_t s);

/* Ends a chunk of which only the first accepted[b] + 1 rows stay: len[b] -= m_b - 1 - accepted[b]
   (m_b = 0: nothing, whatever accepted[b] holds).  The counterpart of lg_begin_chunk after
   lg_verify_draft; the rows' slots are taken by the next tokens.  An accepted[b] outside [0, m_b - 1], an m_b outside [0, max_new] or above
   len[b], or an off[] outside [0, T] sets LG_ERR_CAPACITY on the device and leaves that sequence's
   length.  accepted: device [batch]. */
LG_API lg_status lg_end_chunk(const lg_cache *c, const lg_chunk *ch, const int32_t *accepted,
                              cudaStream_t s);

/* The chunk's rows of one layer of a 4-bit cache as the values that they stand for: for the j-th new
   token of sequence b, t = off[b] + j,
     k_out[t][h][:], v_out[t][h][:] = rows len[b] - m_b + j of kv-head h, s c + lo rounded to bf16
   A chunk of m_b = len[b] reads whole sequences.  k_out, v_out: device [T][H_kv][d] bf16 dense, 16-byte
   aligned; rows of no sequence are left as they were.  LG_ERR_UNSUPPORTED for a cache of another
   dtype. */
LG_API lg_status lg_read_rows(const lg_cache *c, const lg_chunk *ch, int layer, void *k_out,
                              void *v_out, cudaStream_t s);

#ifdef __cplusplus
}
#endif
#endif
