// C ABI of include/lg_chunk.h: host-side validation, frequencies, workspace layout and launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "lg_chunk.h"
#include "lg_chunk_attend.cuh"
#include "lg_internal.h"
#include "lg_q4.cuh"

namespace {

using lg::check_cache;
using lg::check_params;

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// n and m bytes at a and b have some in common
bool overlap(const void *a, uint64_t n, const void *b, uint64_t m) {
  const uint64_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + m && y < x + n;
}

lg_status cuda_status(cudaError_t e) { return e == cudaSuccess ? LG_OK : LG_ERR_CUDA; }

lg_status check_chunk(const lg_cache *c, const lg_chunk *ch) {
  const lg_status st = check_cache(c);
  if (st != LG_OK) return st;
  if (!ch || !ch->off || !aligned(ch->off, 4) || ch->T < 0 || ch->max_new < 0)
    return LG_ERR_INVALID_ARG;
  return LG_OK;
}

lg_status check_rope(const lg_rope_params *p, int d) {
  if (!p) return LG_ERR_INVALID_ARG;
  if (p->layout != LG_ROPE_HALF && p->layout != LG_ROPE_INTERLEAVED) return LG_ERR_INVALID_ARG;
  if (p->scaling < LG_ROPE_PLAIN || p->scaling > LG_ROPE_YARN) return LG_ERR_INVALID_ARG;
  if (p->rot < 16 || p->rot > d || p->rot % 16) return LG_ERR_UNSUPPORTED;
  if (!(p->theta > 1.0) || !isfinite(p->theta)) return LG_ERR_INVALID_ARG;
  if (!(p->mscale > 0.0) || !isfinite(p->mscale)) return LG_ERR_INVALID_ARG;
  if (p->scaling != LG_ROPE_PLAIN && (!(p->factor >= 1.0) || !isfinite(p->factor)))
    return LG_ERR_INVALID_ARG;
  if (p->scaling == LG_ROPE_BANDS &&
      (p->orig_len < 1 || !(p->low > 0.0) || !(p->high > p->low) || !isfinite(p->high)))
    return LG_ERR_INVALID_ARG;
  if (p->scaling == LG_ROPE_YARN && (p->orig_len < 1 || !(p->beta_slow > 0.0) ||
                                     !(p->beta_fast > p->beta_slow) || !isfinite(p->beta_fast)))
    return LG_ERR_INVALID_ARG;
  return LG_OK;
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

// f_i / 2 pi in units of 2^-64 turns
void rope_turns(const lg_rope_params &p, uint64_t *turns) {
  const double rot = p.rot;
  const double theta =
      p.scaling == LG_ROPE_BASE ? p.theta * pow(p.factor, rot / (rot - 2.0)) : p.theta;
  double a = 0.0, span = 1.0;  // YARN's ramp
  if (p.scaling == LG_ROPE_YARN) {
    auto pair_at = [&](double turns_over) {
      return rot * log(p.orig_len / (turns_over * kTwoPi)) / (2.0 * log(theta));
    };
    a = fmax(floor(pair_at(p.beta_fast)), 0.0);
    const double b = fmin(ceil(pair_at(p.beta_slow)), rot - 1.0);
    span = fmax(b - a, 0.001);
  }
  // theta^(-2i/rot) from the powers at i = 1, 2, 4, ..: at most six products, so at most twelve
  // roundings, for a seventh of the time of a pow a pair
  double power[6], f[64];
  for (int k = 0; 1 << k < p.rot / 2; ++k) power[k] = pow(theta, -2.0 * (1 << k) / rot);
  const double inv = p.scaling == LG_ROPE_PLAIN || p.scaling == LG_ROPE_BASE ? 1.0 : 1.0 / p.factor;
  f[0] = 1.0;
  for (int i = 0; i < p.rot / 2; ++i) {
    if (i) {
      int k = 0;
      while (!(i >> k & 1)) ++k;
      f[i] = f[i & (i - 1)] * power[k];
    }
    double w = 1.0;  // the share that keeps its frequency
    if (p.scaling == LG_ROPE_LINEAR) w = 0.0;
    if (p.scaling == LG_ROPE_BANDS)
      w = fmin(fmax((p.orig_len * f[i] / kTwoPi - p.low) / (p.high - p.low), 0.0), 1.0);
    if (p.scaling == LG_ROPE_YARN) w = 1.0 - fmin(fmax((i - a) / span, 0.0), 1.0);
    const double t = (w * f[i] + (1.0 - w) * f[i] * inv) * (0x1p64 / kTwoPi);
    turns[i] = (uint64_t)llrint(t);  // f <= 1: below 2^62
  }
}

lg_status attend_shape(const lg_cache *c, const lg_chunk *ch, int H_q, int max_len) {
  const lg_status st = check_chunk(c, ch);
  if (st != LG_OK) return st;
  if (H_q < 1 || H_q % c->H_kv || max_len < 1) return LG_ERR_INVALID_ARG;
  if (H_q / c->H_kv > 8) return LG_ERR_UNSUPPORTED;
  return LG_OK;
}

size_t part_bytes(const lg::ChunkGrid &g, int d) {
  const size_t n = (size_t)g.ctas * (2 * g.rows * (d + 2) * sizeof(float) + sizeof(lg::ChunkCut));
  return (n + 255) / 256 * 256;
}

lg_status check_rows(const lg_logits *x) {
  if (!x || !x->x) return LG_ERR_INVALID_ARG;
  if (x->dtype != LG_BF16 && x->dtype != LG_F32) return LG_ERR_UNSUPPORTED;
  if (x->batch < 1 || x->V < 1 || x->stride < x->V) return LG_ERR_INVALID_ARG;
  if (x->V > 1 << 20) return LG_ERR_UNSUPPORTED;
  return aligned(x->x, x->dtype == LG_BF16 ? 2 : 4) ? LG_OK : LG_ERR_INVALID_ARG;
}

// lg_chunk_attend over a 4-bit cache: few query rows of a kv-head read the codes themselves
bool q4_few(const lg_chunk *ch, int g) { return (int64_t)ch->max_new * g <= lg::kQ4FewRows; }

// bytes of one layer's keys (or values) in bf16
size_t q4_plane_bytes(const lg_cache *c) {
  return ((size_t)c->H_kv * c->S_total * c->d * 2 + 255) / 256 * 256;
}

size_t q4_chunk_bytes(const lg_cache *c, const lg_chunk *ch, int g, int max_len) {
  if (q4_few(ch, g)) {
    const size_t n = lg::q4_grid(1, c->batch, c->H_kv, g, c->d, ch->max_new, max_len, 0, 0).part_bytes;
    return n > 256 ? n : 256;
  }
  return 2 * q4_plane_bytes(c) + part_bytes(lg::chunk_grid(LG_BF16, c->d, g, ch->max_new), c->d);
}

}  // namespace

extern "C" {

lg_status lg_begin_chunk(const lg_cache *c, const lg_chunk *ch, cudaStream_t s) {
  const lg_status st = check_chunk(c, ch);
  if (st != LG_OK) return st;
  return cuda_status(lg::launch_begin_chunk(*c, *ch, s));
}

lg_status lg_default_rope_params(lg_rope_params *p, int d) {
  if (!p || d < 16) return LG_ERR_INVALID_ARG;
  memset(p, 0, sizeof(*p));
  p->layout = LG_ROPE_HALF;
  p->rot = d;
  p->scaling = LG_ROPE_PLAIN;
  p->orig_len = 8192;
  p->theta = 10000.0;
  p->factor = 1.0;
  p->low = 1.0;
  p->high = 4.0;
  p->beta_fast = 32.0;
  p->beta_slow = 1.0;
  p->mscale = 1.0;
  return LG_OK;
}

lg_status lg_rope_append(const lg_cache *c, const lg_chunk *ch, int layer, const void *q,
                         int64_t q_stride, int H_q, const void *k_new, int64_t k_stride,
                         const void *v_new, int64_t v_stride, const int32_t *pos,
                         const lg_rope_params *rp, void *q_out, const lg_guard_params *p,
                         cudaStream_t s) {
  lg_status st = check_chunk(c, ch);
  if (st != LG_OK) return st;
  if ((st = check_params(p)) != LG_OK) return st;
  if ((st = check_rope(rp, c->d)) != LG_OK) return st;
  if (layer < 0 || layer >= c->L || H_q < 0 || H_q > 65536) return LG_ERR_INVALID_ARG;
  if (ch->T == 0) return LG_OK;
  if (!k_new || !v_new || !pos || (H_q > 0) != (q != nullptr) || (H_q > 0) != (q_out != nullptr))
    return LG_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q_out, 16) ||
      !aligned(pos, 4))
    return LG_ERR_INVALID_ARG;
  const int64_t el = c->dtype == LG_F32 ? 4 : 8;  // elements of 16 bytes
  if (k_stride % el || v_stride % el || k_stride < (int64_t)c->H_kv * c->d ||
      v_stride < (int64_t)c->H_kv * c->d)
    return LG_ERR_INVALID_ARG;
  if (H_q > 0 && (q_stride % el || q_stride < (int64_t)H_q * c->d)) return LG_ERR_INVALID_ARG;
  if (H_q > 0) {  // the rotated queries overwrite none that other threads still read
    const uint64_t es = 16 / el, row = (uint64_t)H_q * c->d * es;
    const uint64_t kv_row = (uint64_t)c->H_kv * c->d * es, last = (uint64_t)(ch->T - 1) * es;
    if (q == q_out ? q_stride != (int64_t)H_q * c->d
                   : overlap(q_out, ch->T * row, q, last * q_stride + row))
      return LG_ERR_INVALID_ARG;
    if (overlap(q_out, ch->T * row, k_new, last * k_stride + kv_row) ||
        overlap(q_out, ch->T * row, v_new, last * v_stride + kv_row))
      return LG_ERR_INVALID_ARG;
  }
  uint64_t turns[64];
  rope_turns(*rp, turns);
  if (c->dtype == LG_Q4)
    return cuda_status(lg::launch_q4_rope_append(
        *c, *ch, layer, q, q_stride, H_q, k_new, k_stride, v_new, v_stride, pos, *rp, turns, q_out,
        c->sketch && p->guard_layer == layer, s));
  return cuda_status(lg::launch_rope_append(*c, *ch, layer, q, q_stride, H_q, k_new, k_stride,
                                            v_new, v_stride, pos, *rp, turns, q_out,
                                            c->sketch && p->guard_layer == layer, s));
}

size_t lg_chunk_workspace_size(const lg_cache *c, const lg_chunk *ch, int H_q, int max_len) {
  if (attend_shape(c, ch, H_q, max_len) != LG_OK) return 0;
  if (c->dtype == LG_Q4) return q4_chunk_bytes(c, ch, H_q / c->H_kv, max_len);
  return part_bytes(lg::chunk_grid(c->dtype, c->d, H_q / c->H_kv, ch->max_new), c->d);
}

lg_status lg_chunk_attend(const lg_cache *c, const lg_chunk *ch, int layer, const void *q, int H_q,
                          float scale, int window, int n_sink, void *out, int max_len, void *ws,
                          size_t ws_bytes, cudaStream_t s) {
  const lg_status st = attend_shape(c, ch, H_q, max_len);
  if (st != LG_OK) return st;
  if (layer < 0 || layer >= c->L || window < 0 || n_sink < 0) return LG_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !isfinite(scale)) return LG_ERR_INVALID_ARG;
  if (c->dtype == LG_BF16 && (int64_t)c->L * c->H_kv * c->S_total >= ((int64_t)1 << 31))
    return LG_ERR_UNSUPPORTED;
  if (c->dtype == LG_Q4 && !q4_few(ch, H_q / c->H_kv) &&
      (int64_t)c->H_kv * c->S_total >= ((int64_t)1 << 31))
    return LG_ERR_UNSUPPORTED;
  if (ch->T == 0 || ch->max_new == 0) return LG_OK;
  if (!q || !out || q == out || !aligned(q, 16) || !aligned(out, 16)) return LG_ERR_INVALID_ARG;
  const int g = H_q / c->H_kv;
  const uint64_t bytes = (uint64_t)ch->T * H_q * c->d * (c->dtype == LG_F32 ? 4 : 2);
  if (c->dtype == LG_Q4) {
    if (!ws || !aligned(ws, 256) || ws_bytes < q4_chunk_bytes(c, ch, g, max_len))
      return LG_ERR_WORKSPACE;
    if (overlap(q, bytes, out, bytes)) return LG_ERR_INVALID_ARG;
    if (q4_few(ch, g)) {
      const lg::Q4Grid grid =
          lg::q4_grid(1, c->batch, c->H_kv, g, c->d, ch->max_new, max_len, window, n_sink);
      if (!lg::q4_grid_fits(1, c->batch, c->H_kv)) return LG_ERR_UNSUPPORTED;
      lg::Q4AttendArgs a = {};
      a.q = q;
      a.out = out;
      a.off = ch->off;
      a.layer0 = layer;
      a.n_layers = 1;
      a.T = ch->T;
      a.max_new = ch->max_new;
      a.max_len = max_len;
      a.shape.window = window;
      a.shape.sink = n_sink;
      lg::q4_fill(a, *c, g, scale, grid, ws);
      return cuda_status(lg::launch_q4_attend(a, c->d, s));
    }
  }
  // many query rows over four bits: a 16-bit layer of the rows' values, then the kernels of such
  lg_cache wide = *c;
  if (c->dtype == LG_Q4) {
    const size_t plane = q4_plane_bytes(c);
    wide.k = ws;
    wide.v = (char *)ws + plane;
    wide.dtype = LG_BF16;
    wide.L = 1;
    const cudaError_t e = lg::launch_q4_expand(*c, *ch, layer, window, n_sink, max_len, wide.k,
                                               wide.v, s);
    if (e != cudaSuccess) return LG_ERR_CUDA;
    ws = (char *)ws + 2 * plane;
    ws_bytes -= 2 * plane;
    layer = 0;
    c = &wide;
  }
  const lg::ChunkGrid grid = lg::chunk_grid(c->dtype, c->d, g, ch->max_new);
  if (!ws || !aligned(ws, 256) || ws_bytes < part_bytes(grid, c->d)) return LG_ERR_WORKSPACE;
  if (overlap(q, bytes, out, bytes)) return LG_ERR_INVALID_ARG;
  lg::ChunkAttendArgs a = {};
  a.K = c->k;
  a.V = c->v;
  a.q = q;
  a.out = out;
  a.seq_off = c->seq_off;
  a.len = c->len;
  a.off = ch->off;
  a.status = c->dev_status;
  a.part = (float *)ws;
  a.S_total = c->S_total;
  a.cache_rows = (int64_t)c->L * c->H_kv * c->S_total;
  a.layer = layer;
  a.batch = c->batch;
  a.H_kv = c->H_kv;
  a.g = g;
  a.T = ch->T;
  a.max_new = ch->max_new;
  a.max_len = max_len;
  a.rows = grid.rows;
  a.qscale = scale * 1.4426950408889634f;
  a.shape.tok = grid.tok;
  a.shape.bn2 = grid.bn2;
  a.shape.window = window;
  a.shape.sink = n_sink;
  return cuda_status(lg::launch_chunk_attend(a, c->dtype, c->d, grid.ctas, s));
}

lg_status lg_end_chunk(const lg_cache *c, const lg_chunk *ch, const int32_t *accepted,
                       cudaStream_t s) {
  const lg_status st = check_chunk(c, ch);
  if (st != LG_OK) return st;
  if (!accepted || !aligned(accepted, 4)) return LG_ERR_INVALID_ARG;
  return cuda_status(lg::launch_end_chunk(*c, *ch, accepted, s));
}

lg_status lg_read_rows(const lg_cache *c, const lg_chunk *ch, int layer, void *k_out, void *v_out,
                       cudaStream_t s) {
  const lg_status st = check_chunk(c, ch);
  if (st != LG_OK) return st;
  if (c->dtype != LG_Q4) return LG_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= c->L) return LG_ERR_INVALID_ARG;
  if (ch->T == 0) return LG_OK;
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return LG_ERR_INVALID_ARG;
  const uint64_t bytes = (uint64_t)ch->T * c->H_kv * c->d * 2;
  if (overlap(k_out, bytes, v_out, bytes)) return LG_ERR_INVALID_ARG;
  return cuda_status(lg::launch_q4_read(*c, *ch, layer, k_out, v_out, s));
}

size_t lg_verify_workspace_size(const lg_logits *x, const lg_chunk *ch) {
  if (check_rows(x) != LG_OK || !ch || ch->T < 0 || ch->T > 65535) return 0;
  const size_t n = lg::verify_ws_bytes(*x, ch->T);
  return n > 16 ? n : 16;
}

lg_status lg_verify_draft(const lg_logits *x, const lg_chunk *ch, int batch, const int32_t *tokens,
                          const lg_logits *draft, const float *temperature, const float *u,
                          const float *r, int32_t *picked, int32_t *accepted, void *ws,
                          size_t ws_bytes, int32_t *dev_status, cudaStream_t s) {
  lg_status st = check_rows(x);
  if (st != LG_OK) return st;
  if (draft && (st = check_rows(draft)) != LG_OK) return st;
  if (!ch || !ch->off || !aligned(ch->off, 4) || ch->T < 0 || ch->max_new < 0 || batch < 1)
    return LG_ERR_INVALID_ARG;
  if (ch->T > 65535 || batch > 1 << 20) return LG_ERR_UNSUPPORTED;
  if (x->batch < ch->T || (draft && (draft->batch < ch->T || draft->V != x->V)))
    return LG_ERR_INVALID_ARG;
  if (!tokens || !u || !r || !picked || !accepted || !aligned(tokens, 4) || !aligned(u, 4) ||
      !aligned(r, 4) || !aligned(temperature, 4) || !aligned(picked, 4) || !aligned(accepted, 4) ||
      !aligned(dev_status, 4))
    return LG_ERR_INVALID_ARG;
  if (!ws || !aligned(ws, 16) || ws_bytes < lg::verify_ws_bytes(*x, ch->T)) return LG_ERR_WORKSPACE;
  // results over anything that is read, or over one another
  const uint64_t n = (uint64_t)ch->T * 4, nb = (uint64_t)batch * 4;
  auto rows = [&](const lg_logits *l) {
    return ch->T ? ((uint64_t)(ch->T - 1) * l->stride + l->V) * (l->dtype == LG_BF16 ? 2 : 4) : 0;
  };
  auto taken = [&](const void *p, uint64_t bytes) {
    return p && (overlap(picked, n, p, bytes) || overlap(accepted, nb, p, bytes));
  };
  if (overlap(picked, n, accepted, nb) || taken(tokens, n) || taken(u, n) || taken(r, nb) ||
      taken(temperature, nb) || taken(ch->off, nb + 4) || taken(x->x, rows(x)) ||
      (draft && taken(draft->x, rows(draft))) || taken(ws, lg::verify_ws_bytes(*x, ch->T)))
    return LG_ERR_INVALID_ARG;
  return cuda_status(lg::launch_verify(*x, *ch, batch, tokens, draft, temperature, u, r, picked,
                                       accepted, ws, dev_status, s));
}

lg_status lg_count_tokens(const int32_t *tokens, const int32_t *off, int T, int batch, int V,
                          int generated, uint32_t *seen, int32_t *counts, int32_t *dev_status,
                          cudaStream_t s) {
  if (!tokens || !seen || !counts || T < 0 || batch < 1 || V < 1 || (!off && T != batch))
    return LG_ERR_INVALID_ARG;
  if (!aligned(tokens, 4) || !aligned(off, 4) || !aligned(seen, 4) || !aligned(counts, 4) ||
      !aligned(dev_status, 4))
    return LG_ERR_INVALID_ARG;
  return cuda_status(lg::launch_count_tokens(tokens, off, T, batch, V, generated, seen, counts,
                                             dev_status, s));
}

lg_status lg_pick_token(const lg_logits *x, const uint32_t *seen, const int32_t *counts,
                        const float *penalty, const lg_bias *bias, const uint32_t *allowed,
                        int32_t *tokens, float *pmax, void *logits_out, int32_t *dev_status,
                        cudaStream_t s) {
  if (!x || !x->x || !tokens || !pmax) return LG_ERR_INVALID_ARG;
  if (x->dtype != LG_BF16 && x->dtype != LG_F32) return LG_ERR_UNSUPPORTED;
  const size_t es = x->dtype == LG_BF16 ? 2 : 4;
  if (x->batch < 1 || x->V < 1 || x->stride < x->V) return LG_ERR_INVALID_ARG;
  if (x->V > 1 << 20 || x->batch > 1 << 20) return LG_ERR_UNSUPPORTED;
  if (!aligned(x->x, es) || !aligned(logits_out, es)) return LG_ERR_INVALID_ARG;
  if (!aligned(seen, 4) || !aligned(counts, 4) || !aligned(allowed, 4) || !aligned(tokens, 4) ||
      !aligned(pmax, 4) || !aligned(dev_status, 4))
    return LG_ERR_INVALID_ARG;
  if ((seen == nullptr) != (counts == nullptr) || (seen == nullptr) != (penalty == nullptr) ||
      !aligned(penalty, 16))
    return LG_ERR_INVALID_ARG;
  if (bias && (!bias->off || !bias->id || !bias->val || !aligned(bias->off, 4) ||
               !aligned(bias->id, 4) || !aligned(bias->val, 4)))
    return LG_ERR_INVALID_ARG;
  if (logits_out && logits_out != x->x) {  // rows beside x's in one buffer, or apart from them
    const uint64_t step = (uint64_t)x->stride * es, row = (uint64_t)x->V * es;
    const uint64_t all = (uint64_t)(x->batch - 1) * step + row;
    const uint64_t from = (uintptr_t)x->x, to = (uintptr_t)logits_out;
    const uint64_t d = to > from ? (to - from) % step : (step - (from - to) % step) % step;
    const bool beside = d >= row && d + row <= step;
    if (overlap(x->x, all, logits_out, all) && !beside) return LG_ERR_INVALID_ARG;
  }
  return cuda_status(lg::launch_pick_token(*x, seen, counts, penalty, bias, allowed, tokens, pmax,
                                           logits_out, dev_status, s));
}

}  // extern "C"
