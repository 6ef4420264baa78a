// Host side of the layer norm and cross-attention entry points of include/sva.h:
// argument validation and dispatch.  Every check runs before any HIP call.
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sva.h"
#include "api_checks.h"
#include "cross_args.h"
#include "norm_args.h"
#include "sva_internal.h"

namespace {

using namespace sva::api;

// What a call writes has to lie apart from all that it reads and writes beside it, as it is
// written while other workgroups still read: the first `written` of `count`.
bool shares(const Tensor* const* all, int written, int count) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < count; ++j)
      if (all[i]->v.p && all[j]->v.p && meet(*all[i], *all[j])) return true;
  return false;
}

// ---- layer norm ----

// One tensor [B, N, C] as a tensor of one head.
int check_rows3(const sva_rows* r, int64_t B, int64_t N, int64_t C, size_t item, bool output, Tensor* t) {
  if (!r) return SVA_ERR_INVALID_ARG;
  const sva_heads h = {r->data, 1, r->stride_b, 0, r->stride_n};
  return check_heads(&h, B, N, C, item, false, output, t);
}

int check_norm(const sva_layer_norm_params* p) {
  if (!p || p->batch < 1 || p->tokens < 1 || p->channels < 1) return SVA_ERR_INVALID_ARG;
  if (!good_dtype(p->dtype) || !good_dtype(p->weight_dtype)) return SVA_ERR_INVALID_ARG;
  if (!((float)p->eps >= FLT_MIN && (float)p->eps <= FLT_MAX)) return SVA_ERR_INVALID_ARG;
  if (p->weight_stride_b < 0 || p->bias_stride_b < 0) return SVA_ERR_INVALID_ARG;
  if (p->channels > sva::kNormMaxChannels) return SVA_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->tokens > INT32_MAX - (1 << 20)) return SVA_ERR_SHAPE;
  if (p->weight_stride_b > (int64_t)1 << 40 || p->bias_stride_b > (int64_t)1 << 40) return SVA_ERR_SHAPE;
  return SVA_OK;
}

// Where weights are shared, entries whose rows follow each other at one pitch are one entry.
bool one_run(const Tensor& t, int64_t B, int64_t N) { return B == 1 || N == 1 || t.v.sb == N * t.v.sn; }

sva::RowsView view(const Tensor& t, bool joined, int64_t N) {
  return {t.v.p, joined ? 0 : t.v.sb, joined && N == 1 ? t.v.sb : t.v.sn};
}

// Sizes as the kernels take them; `joined`: all entries as one.
int norm_sizes(const sva_layer_norm_params* p, bool joined, bool grad, sva::NormArgs* a, sva::NormShape* s) {
  a->B = joined ? 1 : p->batch;
  a->N = joined ? p->batch * p->tokens : p->tokens;
  a->C = p->channels;
  *s = sva::norm_shape(a->B, a->N, a->C, grad, joined || p->per_entry != 0);
  // a launch has 2^22 workgroups at most, and fewer than 2^32 threads
  const int64_t wgs = (int64_t)a->B * s->parts;
  if (wgs > 1 << 22 || wgs * s->threads >= (int64_t)1 << 32) return SVA_ERR_SHAPE;
  a->parts = s->parts;
  return SVA_OK;
}

void norm_weights(const sva_layer_norm_params* p, const void* weight, const void* bias, sva::NormArgs* a) {
  a->w = weight;
  a->bias = bias;
  a->w_b = p->per_entry ? p->weight_stride_b : 0;
  a->bias_b = p->per_entry ? p->bias_stride_b : 0;
  a->w_bf16 = p->weight_dtype == SVA_BF16;
  a->unit = p->unit_offset ? 1.0f : 0.0f;
  a->eps = (float)p->eps;
  a->f32 = p->dtype == SVA_F32;
}

Tensor weight_of(const sva_layer_norm_params* p, const void* w, int64_t stride_b) {
  const int64_t item = (int64_t)item_of(p->weight_dtype);
  const bool rows = p->per_entry && p->batch > 1;
  return runs_of(w, rows ? p->batch : 1, rows ? stride_b * item : 0, p->channels * item);
}
Tensor stat_of(const sva_layer_norm_params* p, const float* s) { return runs_of(s, 1, 0, (int64_t)p->batch * p->tokens * 4); }
Tensor sum_of(const sva_layer_norm_params* p, const float* s) {
  return runs_of(s, 1, 0, (int64_t)(p->per_entry ? p->batch : 1) * p->channels * 4);
}

// ---- cross attention ----

int check_cross(const sva_cross* p) {
  if (!p) return SVA_ERR_INVALID_ARG;
  if (p->batch < 1 || p->heads < 1 || p->kv_heads < 1 || p->queries < 1 || p->keys < 1) return SVA_ERR_INVALID_ARG;
  if (p->softmax_scale != p->softmax_scale || isinf(p->softmax_scale)) return SVA_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 112 && p->head_dim != 128) return SVA_ERR_UNSUPPORTED;
  if (p->heads % p->kv_heads != 0) return SVA_ERR_SHAPE;
  // rows of queries and of keys are counted in 32 bits
  int64_t rows, keys;
  if (__builtin_mul_overflow((int64_t)p->batch * p->heads, (int64_t)p->queries, &rows) || rows > INT32_MAX - (1 << 16))
    return SVA_ERR_SHAPE;
  if (__builtin_mul_overflow((int64_t)p->batch * p->kv_heads, (int64_t)p->keys, &keys) || keys > INT32_MAX - (1 << 16))
    return SVA_ERR_SHAPE;
  return SVA_OK;
}

int cross_sizes(const sva_cross* p, bool mask, bool grad, sva::CrossArgs* a, sva::CrossShape* s) {
  a->B = p->batch;
  a->H = p->heads;
  a->Hkv = p->kv_heads;
  a->G = p->heads / p->kv_heads;
  a->N = p->queries;
  a->M = p->keys;
  a->R = a->G * a->N;
  a->D = p->head_dim;
  const double c = p->softmax_scale > 0.0 ? p->softmax_scale : 1.0 / sqrt((double)p->head_dim);
  a->scale = (float)c;
  a->scale_log2 = (float)(c * 1.4426950408889634074);
  // zero would make a hidden key's logit 0 * -inf, infinity every other's
  if (!(a->scale >= FLT_MIN && a->scale_log2 <= FLT_MAX)) return SVA_ERR_INVALID_ARG;
  *s = grad ? sva::cross_grad_shape(a->B, a->Hkv, a->G, a->N, a->M, a->D, mask)
            : sva::cross_shape(a->B, a->Hkv, a->G, a->N, a->M, a->D, mask, false);
  a->tiles = s->tiles;
  a->run = s->run;
  a->splits = s->splits;
  a->key_tiles = s->key_tiles;
  a->row_splits = s->row_splits;
  // a launch has fewer than 2^32 threads, 256 (join: a row each) a workgroup
  const int64_t heads = (int64_t)a->B * a->Hkv, most = ((int64_t)1 << 24) - 1;
  const int64_t wgs = heads * ((s->tiles + s->run - 1) / s->run) * s->splits, kv_wgs = heads * s->key_tiles * s->row_splits;
  if (wgs > most || kv_wgs > most || (s->splits > 1 && heads * a->R > most)) return SVA_ERR_SHAPE;
  if (mask && a->B > most / 4) return SVA_ERR_SHAPE;      // (an entry's mask: 1,024 threads)
  a->wgs = (int)wgs;
  a->kv_wgs = (int)kv_wgs;
  return SVA_OK;
}

int check_hidden(const sva_cross* p, const int32_t* lengths, const uint8_t* mask, int64_t mask_stride_b, sva::CrossArgs* a) {
  if (mask_stride_b < 0) return SVA_ERR_INVALID_ARG;
  if (mask && p->batch > 1 && mask_stride_b > (int64_t)1 << 40) return SVA_ERR_SHAPE;
  if (lengths && !aligned(lengths, 4)) return SVA_ERR_ALIGNMENT;
  a->lens = lengths;
  a->mask = mask;
  a->mask_b = mask_stride_b;
  return SVA_OK;
}

// One tensor of heads: of queries, or of keys.
int check_cross_tensor(const sva_cross* p, const sva_heads* h, bool keys, bool output, Tensor* t) {
  const int st = check_heads(h, p->batch, keys ? p->keys : p->queries, p->head_dim, 2, true, output, t);
  if (st != SVA_OK) return st;
  return t->v.heads == (keys ? p->kv_heads : p->heads) ? SVA_OK : SVA_ERR_SHAPE;
}

int check_workspace(void* workspace, size_t bytes, size_t need) {
  if (need == 0) return SVA_OK;
  if (!workspace) return SVA_ERR_INVALID_ARG;
  if (bytes < need) return SVA_ERR_SHAPE;
  return aligned(workspace, 256) ? SVA_OK : SVA_ERR_ALIGNMENT;
}

Tensor lengths_of(const sva_cross* p, const int32_t* lengths) { return runs_of(lengths, 1, 0, (int64_t)p->batch * 4); }
Tensor mask_of(const sva_cross* p, const uint8_t* mask, int64_t stride_b) {
  return runs_of(mask, p->batch, p->batch > 1 ? stride_b : 0, p->keys);
}
Tensor lse_of(const sva_cross* p, const float* lse) {
  return runs_of(lse, 1, 0, (int64_t)p->batch * p->heads * p->queries * 4);
}

void place_workspace(void* workspace, const sva::CrossShape& s, sva::CrossArgs* a) {
  unsigned char* w = static_cast<unsigned char*>(workspace);
  a->bits = reinterpret_cast<uint32_t*>(w + s.bits_at);
  a->seen = reinterpret_cast<int32_t*>(w + s.seen_at);
  a->stat = reinterpret_cast<float2*>(w + s.stat_at);
  a->stat_l = reinterpret_cast<float*>(w + s.stat_l_at);
  a->part = reinterpret_cast<float*>(w + s.part_at);
  a->part_kv = reinterpret_cast<float*>(w + s.part_kv_at);
}

}  // namespace

extern "C" {

int sva_layer_norm(const sva_layer_norm_params* p, const sva_rows* x, const void* weight, const void* bias,
                   const sva_rows* y, float* mean, float* rstd, void* stream) {
  int st = check_norm(p);
  if (st != SVA_OK) return st;
  const int64_t B = p->batch, N = p->tokens, C = p->channels;
  const size_t item = item_of(p->dtype), w_item = item_of(p->weight_dtype);
  Tensor tx, ty;
  if ((st = check_rows3(x, B, N, C, item, false, &tx)) != SVA_OK) return st;
  if ((st = check_rows3(y, B, N, C, item, true, &ty)) != SVA_OK) return st;
  if (!same(tx, ty, B, N) && !apart(tx, ty)) return SVA_ERR_INVALID_ARG;
  if ((weight && !aligned(weight, w_item)) || (bias && !aligned(bias, w_item)) || !aligned(mean, 4) || !aligned(rstd, 4))
    return SVA_ERR_ALIGNMENT;
  const bool joined = !p->per_entry && one_run(tx, B, N) && one_run(ty, B, N);
  sva::NormArgs a{};
  sva::NormShape s;
  if ((st = norm_sizes(p, joined, false, &a, &s)) != SVA_OK) return st;
  const Tensor tw = weight_of(p, weight, p->weight_stride_b), tb = weight_of(p, bias, p->bias_stride_b);
  const Tensor tm = stat_of(p, mean), tr = stat_of(p, rstd);
  const Tensor *stats[] = {&tm, &tr, &ty, &tx, &tw, &tb}, *result[] = {&ty, &tw, &tb};
  if (shares(stats, 2, 6) || shares(result, 1, 3)) return SVA_ERR_INVALID_ARG;
  norm_weights(p, weight, bias, &a);
  a.x = view(tx, joined, N);
  a.y = view(ty, joined, N);
  a.mean = mean;
  a.rstd = rstd;
  a.aligned = C % 8 == 0 && tx.align == 16 && ty.align == 16;
  return hip_status(sva::launch_layer_norm(a, s, static_cast<hipStream_t>(stream)));
}

// The most that any strides need: entries apart (one row each is a pitch of its own), or as one.
int sva_layer_norm_backward_workspace(const sva_layer_norm_params* p, size_t* bytes) {
  if (!bytes) return SVA_ERR_INVALID_ARG;
  int st = check_norm(p);
  if (st != SVA_OK) return st;
  sva::NormArgs a{};
  sva::NormShape s;
  size_t most = 0;
  const int first = !p->per_entry && (p->batch == 1 || p->tokens == 1);
  for (int joined = first; joined <= (p->per_entry ? 0 : 1); ++joined) {
    st = norm_sizes(p, joined != 0, true, &a, &s);       // (as one, any sizes will do)
    if (st == SVA_OK) most = std::max(most, s.ws_bytes);
  }
  if (st != SVA_OK) return st;
  *bytes = most;
  return SVA_OK;
}

int sva_layer_norm_backward(const sva_layer_norm_params* p, const sva_rows* dy, const sva_rows* x, const void* weight,
                            const float* mean, const float* rstd, void* workspace, size_t workspace_bytes,
                            const sva_rows* dx, float* dweight, float* dbias, void* stream) {
  int st = check_norm(p);
  if (st != SVA_OK) return st;
  if (!mean || !rstd) return SVA_ERR_INVALID_ARG;
  const int64_t B = p->batch, N = p->tokens, C = p->channels;
  const size_t item = item_of(p->dtype);
  Tensor tx, tg, to;
  if ((st = check_rows3(dy, B, N, C, item, false, &tg)) != SVA_OK) return st;
  if ((st = check_rows3(x, B, N, C, item, false, &tx)) != SVA_OK) return st;
  if ((st = check_rows3(dx, B, N, C, item, true, &to)) != SVA_OK) return st;
  if ((!same(tx, to, B, N) && !apart(tx, to)) || (!same(tg, to, B, N) && !apart(tg, to))) return SVA_ERR_INVALID_ARG;
  if ((weight && !aligned(weight, item_of(p->weight_dtype))) || !aligned(mean, 4) || !aligned(rstd, 4) ||
      !aligned(dweight, 4) || !aligned(dbias, 4))
    return SVA_ERR_ALIGNMENT;
  const bool joined = !p->per_entry && one_run(tx, B, N) && one_run(tg, B, N) && one_run(to, B, N);
  sva::NormArgs a{};
  sva::NormShape s;
  if ((st = norm_sizes(p, joined, true, &a, &s)) != SVA_OK) return st;
  const bool sums = dweight || dbias;
  if (sums && (st = check_workspace(workspace, workspace_bytes, s.ws_bytes)) != SVA_OK) return st;
  const Tensor tw = weight_of(p, weight, p->weight_stride_b), tm = stat_of(p, mean), tr = stat_of(p, rstd);
  const Tensor tdw = sum_of(p, dweight), tdb = sum_of(p, dbias);
  const Tensor ts = runs_of(sums && s.ws_bytes ? workspace : nullptr, 1, 0, (int64_t)s.ws_bytes);
  const Tensor *all[] = {&tdw, &tdb, &ts, &to, &tg, &tx, &tw, &tm, &tr}, *result[] = {&to, &tw, &tm, &tr};
  if (shares(all, 3, 9) || shares(result, 1, 4)) return SVA_ERR_INVALID_ARG;
  norm_weights(p, weight, nullptr, &a);
  a.x = view(tx, joined, N);
  a.dy = view(tg, joined, N);
  a.y = view(to, joined, N);
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.partial = sums && s.ws_bytes ? static_cast<float*>(workspace) : nullptr;
  a.dw = dweight;
  a.db = dbias;
  a.aligned = C % 8 == 0 && tx.align == 16 && tg.align == 16 && to.align == 16;
  return hip_status(sva::launch_layer_norm_grad(a, s, p->per_entry ? p->batch : 1, static_cast<hipStream_t>(stream)));
}

int sva_cross_attention_workspace(const sva_cross* p, int32_t masked, size_t* bytes) {
  if (!bytes) return SVA_ERR_INVALID_ARG;
  int st = check_cross(p);
  if (st != SVA_OK) return st;
  sva::CrossArgs a{};
  sva::CrossShape s;
  if ((st = cross_sizes(p, masked != 0, false, &a, &s)) != SVA_OK) return st;
  *bytes = s.ws_bytes;
  return SVA_OK;
}

int sva_cross_attention(const sva_cross* p, const sva_heads* q, const sva_heads* k, const sva_heads* v,
                        const int32_t* lengths, const uint8_t* mask, int64_t mask_stride_b, void* workspace,
                        size_t workspace_bytes, const sva_heads* out, float* lse, void* stream) {
  int st = check_cross(p);
  if (st != SVA_OK) return st;
  sva::CrossArgs a{};
  sva::CrossShape s;
  if ((st = cross_sizes(p, mask != nullptr, false, &a, &s)) != SVA_OK) return st;
  if ((st = check_hidden(p, lengths, mask, mask_stride_b, &a)) != SVA_OK) return st;
  Tensor tq, tk, tv, to;
  if ((st = check_cross_tensor(p, q, false, false, &tq)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, k, true, false, &tk)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, v, true, false, &tv)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, out, false, true, &to)) != SVA_OK) return st;
  if (!aligned(lse, 4)) return SVA_ERR_ALIGNMENT;
  if ((st = check_workspace(workspace, workspace_bytes, s.ws_bytes)) != SVA_OK) return st;
  const Tensor tl = lse_of(p, lse), tn = lengths_of(p, lengths), tm = mask_of(p, mask, mask_stride_b);
  const Tensor tw = runs_of(s.ws_bytes ? workspace : nullptr, 1, 0, (int64_t)s.ws_bytes);
  const Tensor* all[] = {&to, &tl, &tw, &tq, &tk, &tv, &tn, &tm};
  if (shares(all, 3, 8)) return SVA_ERR_INVALID_ARG;
  a.q = tq.v;
  a.k = tk.v;
  a.v = tv.v;
  a.out = to.v;
  a.lse = lse;
  place_workspace(workspace, s, &a);
  return hip_status(sva::launch_cross_attention(a, s, static_cast<hipStream_t>(stream)));
}

int sva_cross_attention_backward_workspace(const sva_cross* p, int32_t masked, size_t* bytes) {
  if (!bytes) return SVA_ERR_INVALID_ARG;
  int st = check_cross(p);
  if (st != SVA_OK) return st;
  sva::CrossArgs a{};
  sva::CrossShape s;
  if ((st = cross_sizes(p, masked != 0, true, &a, &s)) != SVA_OK) return st;
  *bytes = s.ws_bytes;
  return SVA_OK;
}

int sva_cross_attention_backward(const sva_cross* p, const sva_heads* dout, const sva_heads* q, const sva_heads* k,
                                 const sva_heads* v, const sva_heads* out, const float* lse, const int32_t* lengths,
                                 const uint8_t* mask, int64_t mask_stride_b, void* workspace, size_t workspace_bytes,
                                 const sva_heads* dq, const sva_heads* dk, const sva_heads* dv, void* stream) {
  int st = check_cross(p);
  if (st != SVA_OK) return st;
  if (!lse) return SVA_ERR_INVALID_ARG;
  sva::CrossArgs a{};
  sva::CrossShape s;
  if ((st = cross_sizes(p, mask != nullptr, true, &a, &s)) != SVA_OK) return st;
  if ((st = check_hidden(p, lengths, mask, mask_stride_b, &a)) != SVA_OK) return st;
  Tensor tg, tq, tk, tv, to, dtq, dtk, dtv;
  if ((st = check_cross_tensor(p, dout, false, false, &tg)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, q, false, false, &tq)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, k, true, false, &tk)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, v, true, false, &tv)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, out, false, false, &to)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, dq, false, true, &dtq)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, dk, true, true, &dtk)) != SVA_OK) return st;
  if ((st = check_cross_tensor(p, dv, true, true, &dtv)) != SVA_OK) return st;
  if (!aligned(lse, 4)) return SVA_ERR_ALIGNMENT;
  if ((st = check_workspace(workspace, workspace_bytes, s.ws_bytes)) != SVA_OK) return st;
  const Tensor tl = lse_of(p, lse), tn = lengths_of(p, lengths), tm = mask_of(p, mask, mask_stride_b);
  const Tensor tw = runs_of(s.ws_bytes ? workspace : nullptr, 1, 0, (int64_t)s.ws_bytes);
  const Tensor* all[] = {&dtq, &dtk, &dtv, &tw, &tg, &tq, &tk, &tv, &to, &tl, &tn, &tm};
  if (shares(all, 4, 12)) return SVA_ERR_INVALID_ARG;
  a.dout = tg.v;
  a.q = tq.v;
  a.k = tk.v;
  a.v = tv.v;
  a.out = to.v;
  a.dq = dtq.v;
  a.dk = dtk.v;
  a.dv = dtv.v;
  a.lse = const_cast<float*>(lse);
  place_workspace(workspace, s, &a);
  return hip_status(sva::launch_cross_attention_grad(a, s, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
