// Host side of the rotary, cache and cache-attention entry points of
// include/sva.h: argument validation and dispatch.  Every check runs before any
// HIP call.
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sva.h"
#include "sva_internal.h"

namespace {

using sva::HeadsView;

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? SVA_OK : SVA_ERR_HIP; }

// One strided tensor [B, heads, N, D]: its view, and the bytes from its first
// element to behind its last.
struct Tensor {
  HeadsView v;
  size_t span;
  int align;                     // what data and strides are multiples of: 16, 8, 4 or 2 bytes
};

int check_heads(const sva_heads* h, int64_t B, int64_t N, int64_t D, size_t item, bool wide, bool output, Tensor* t) {
  if (!h || !h->data || h->heads < 1) return SVA_ERR_INVALID_ARG;
  if (h->stride_b < 0 || h->stride_h < 0 || h->stride_n < 0) return SVA_ERR_INVALID_ARG;
  struct Dim {
    int64_t size, stride;
  };
  // a dimension of one has no stride
  Dim dims[3] = {{B, B > 1 ? h->stride_b : 0}, {h->heads, h->heads > 1 ? h->stride_h : 0}, {N, N > 1 ? h->stride_n : 0}};
  int64_t span = D;
  for (const Dim& d : dims) {
    int64_t x;
    if (__builtin_mul_overflow(d.size - 1, d.stride, &x) || __builtin_add_overflow(span, x, &span)) return SVA_ERR_SHAPE;
  }
  if (span > ((int64_t)1 << 58)) return SVA_ERR_SHAPE;
  int align = 16;
  auto fits = [&](int n) {
    bool all = aligned(h->data, n);
    for (const Dim& d : dims) all = all && d.stride * (int64_t)item % n == 0;
    return all;
  };
  while (align > (int)item && !fits(align)) align /= 2;
  if (!aligned(h->data, item) || (wide && align < 16)) return SVA_ERR_ALIGNMENT;
  if (output) {                  // rows must not overlap
    std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
    int64_t reach = D;
    for (const Dim& d : dims) {
      if (d.size == 1) continue;
      if (d.stride < reach) return SVA_ERR_INVALID_ARG;
      reach += (d.size - 1) * d.stride;
    }
  }
  t->v.p = h->data;
  t->v.sb = h->stride_b;
  t->v.sh = h->stride_h;
  t->v.sn = h->stride_n;
  t->v.heads = h->heads;
  t->span = (size_t)span * item;
  t->align = align;
  return SVA_OK;
}

bool apart(const Tensor& x, const Tensor& y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.v.p), b = reinterpret_cast<uintptr_t>(y.v.p);
  return a + x.span <= b || b + y.span <= a;
}

bool same(const Tensor& x, const Tensor& y, int64_t B, int64_t N) {
  return x.v.p == y.v.p && (B == 1 || x.v.sb == y.v.sb) && (x.v.heads == 1 || x.v.sh == y.v.sh) &&
         (N == 1 || x.v.sn == y.v.sn);
}

bool good_dtype(int32_t t) { return t == SVA_BF16 || t == SVA_F32; }
size_t item_of(int32_t t) { return t == SVA_F32 ? 4 : 2; }

int check_cache(const sva_cache* c, bool pointers, sva::CacheView* out) {
  if (!c) return SVA_ERR_INVALID_ARG;
  if (c->format != SVA_CACHE_BF16 && c->format != SVA_CACHE_E4M3 && c->format != SVA_CACHE_INT8)
    return SVA_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->kv_heads < 1) return SVA_ERR_INVALID_ARG;
  int log2 = 4;
  while (log2 < 8 && c->page_size != 1 << log2) ++log2;
  if (c->page_size != 1 << log2) return SVA_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 112 && c->head_dim != 128) return SVA_ERR_UNSUPPORTED;
  if ((int64_t)c->num_pages * c->page_size > INT32_MAX || c->kv_heads > 65536) return SVA_ERR_SHAPE;
  if (pointers) {
    if (!c->k || !c->v) return SVA_ERR_INVALID_ARG;
    if (c->format != SVA_CACHE_BF16 && (!c->k_scale || !c->v_scale)) return SVA_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return SVA_ERR_ALIGNMENT;
    if (c->format != SVA_CACHE_BF16 && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))) return SVA_ERR_ALIGNMENT;
  }
  out->k = c->k;
  out->v = c->v;
  out->ks = c->k_scale;
  out->vs = c->v_scale;
  out->format = c->format;       // the enums agree
  out->num_pages = c->num_pages;
  out->heads = c->kv_heads;
  out->log2_page = log2;
  out->D = c->head_dim;
  return SVA_OK;
}
static_assert((int)SVA_CACHE_BF16 == sva::kCacheBf16 && (int)SVA_CACHE_E4M3 == sva::kCacheE4m3 &&
              (int)SVA_CACHE_INT8 == sva::kCacheInt8, "cache formats");

int check_rows(const sva_cache* cache, int32_t batch, int32_t tokens, int32_t dtype, const int32_t* slots,
               int64_t slots_stride_b, const sva_heads* k, const sva_heads* v, bool output, sva::CacheRowsArgs* a) {
  int st = check_cache(cache, true, &a->c);
  if (st != SVA_OK) return st;
  if (batch < 1 || tokens < 1 || !good_dtype(dtype) || !slots || slots_stride_b < 0) return SVA_ERR_INVALID_ARG;
  if ((int64_t)batch * tokens > INT32_MAX) return SVA_ERR_SHAPE;
  // workgroups: at least 16 tokens of four heads each
  if (((int64_t)batch * tokens + 15) / 16 * ((cache->kv_heads + 3) / 4) > INT32_MAX) return SVA_ERR_SHAPE;
  if (batch > 1 && slots_stride_b > (int64_t)1 << 40) return SVA_ERR_SHAPE;
  if (!aligned(slots, 4)) return SVA_ERR_ALIGNMENT;
  Tensor tk, tv;
  const int D = cache->head_dim;
  if ((st = check_heads(k, batch, tokens, D, item_of(dtype), true, output, &tk)) != SVA_OK) return st;
  if ((st = check_heads(v, batch, tokens, D, item_of(dtype), true, output, &tv)) != SVA_OK) return st;
  if (tk.v.heads != cache->kv_heads || tv.v.heads != cache->kv_heads) return SVA_ERR_SHAPE;
  if (output && tk.v.p == tv.v.p) return SVA_ERR_INVALID_ARG;
  a->k = tk.v;
  a->v = tv.v;
  a->slots = slots;
  a->slots_b = slots_stride_b;
  a->B = batch;
  a->N = tokens;
  a->f32 = dtype == SVA_F32;
  return SVA_OK;
}

int check_query(const sva_cache* cache, bool pointers, const sva_cache_query* q, sva::CacheAttnArgs* a) {
  const int st = check_cache(cache, pointers, &a->c);
  if (st != SVA_OK) return st;
  if (!q) return SVA_ERR_INVALID_ARG;
  if (q->batch < 1 || q->heads < 1 || q->queries < 1 || q->max_pages < 1) return SVA_ERR_INVALID_ARG;
  if (!good_dtype(q->out_dtype)) return SVA_ERR_INVALID_ARG;
  if (!(q->softmax_scale == q->softmax_scale) || isinf(q->softmax_scale)) return SVA_ERR_INVALID_ARG;
  if (q->heads % cache->kv_heads != 0) return SVA_ERR_SHAPE;
  if (q->batch > 65536 || q->heads > 65536) return SVA_ERR_SHAPE;
  if (q->queries > SVA_CACHE_MAX_QUERIES) return SVA_ERR_UNSUPPORTED;
  if ((int64_t)q->max_pages * cache->page_size > INT32_MAX - 256) return SVA_ERR_SHAPE;
  a->B = q->batch;
  a->H = q->heads;
  a->G = q->heads / cache->kv_heads;
  a->T = q->queries;
  a->max_pages = q->max_pages;
  // 16-row tiles of all segments, each with four workgroups where results are joined
  if ((int64_t)a->B * cache->kv_heads * (((int64_t)a->G * a->T + 63) / 64) * 16 > INT32_MAX) return SVA_ERR_SHAPE;
  const double c = q->softmax_scale > 0.0 ? q->softmax_scale : 1.0 / sqrt((double)cache->head_dim);
  a->scale_log2 = (float)(c * 1.4426950408889634074);
  // zero would make a masked key's logit 0 * -inf, infinity every other's
  if (!(a->scale_log2 >= FLT_MIN && a->scale_log2 <= FLT_MAX)) return SVA_ERR_INVALID_ARG;
  a->out_f32 = q->out_dtype == SVA_F32;
  return SVA_OK;
}

}  // namespace

extern "C" {

int sva_rotary_frequencies(const sva_rotary_spec* s, double* freq, double* magnitude) {
  if (!s || !freq || !magnitude) return SVA_ERR_INVALID_ARG;
  if (s->rot_dim < 2 || s->rot_dim > 512 || s->rot_dim % 2 != 0) return SVA_ERR_INVALID_ARG;
  if (s->scaling < SVA_ROTARY_PLAIN || s->scaling > SVA_ROTARY_YARN) return SVA_ERR_INVALID_ARG;
  if (!isfinite(s->base) || s->base <= 1.0 || !isfinite(s->magnitude)) return SVA_ERR_INVALID_ARG;
  const bool scaled = s->scaling != SVA_ROTARY_PLAIN, parts = s->scaling == SVA_ROTARY_YARN;
  if (scaled && (!isfinite(s->factor) || s->factor < 1.0)) return SVA_ERR_INVALID_ARG;
  if (parts && (!isfinite(s->original_len) || s->original_len <= 0.0 || !isfinite(s->beta_fast) ||
                !isfinite(s->beta_slow) || s->beta_slow < 0.0 || s->beta_fast <= s->beta_slow))
    return SVA_ERR_INVALID_ARG;
  const double f = scaled ? s->factor : 1.0;
  double base = s->base;
  if (s->scaling == SVA_ROTARY_NTK && s->rot_dim > 2) base *= pow(f, s->rot_dim / (s->rot_dim - 2.0));
  if (!isfinite(base)) return SVA_ERR_INVALID_ARG;
  for (int i = 0; i < s->rot_dim / 2; ++i) {
    double w = pow(base, -2.0 * i / s->rot_dim);
    if (s->scaling == SVA_ROTARY_LINEAR) w /= f;
    if (parts) {
      const double turns = s->original_len * w / 6.283185307179586476925286766559;
      const double keep = std::min(1.0, std::max(0.0, (turns - s->beta_slow) / (s->beta_fast - s->beta_slow)));
      w = (1.0 - keep) * w / f + keep * w;
    }
    freq[i] = w;
  }
  *magnitude = s->magnitude > 0.0 ? s->magnitude : (parts ? 0.1 * log(f) + 1.0 : 1.0);
  return SVA_OK;
}

int sva_rotary(const sva_rotary_params* p, const double* freq, const int32_t* positions, int64_t pos_stride_b,
               const sva_heads* q_in, const sva_heads* q_out, const sva_heads* k_in, const sva_heads* k_out,
               void* stream) {
  if (!p || !freq || !positions || !q_in || !q_out || (!k_in) != (!k_out)) return SVA_ERR_INVALID_ARG;
  if (p->batch < 1 || p->tokens < 1 || p->head_dim < 2 || p->rot_dim < 2 || p->rot_dim % 2 != 0 ||
      p->rot_dim > p->head_dim)
    return SVA_ERR_INVALID_ARG;
  if (p->layout != SVA_ROTARY_HALF && p->layout != SVA_ROTARY_INTERLEAVED) return SVA_ERR_INVALID_ARG;
  if (!good_dtype(p->dtype) || !isfinite(p->magnitude) || pos_stride_b < 0) return SVA_ERR_INVALID_ARG;
  if (p->head_dim > 1024 || p->rot_dim > 512) return SVA_ERR_UNSUPPORTED;
  const int64_t B = p->batch, N = p->tokens, D = p->head_dim;
  if (B * N > INT32_MAX || (B > 1 && pos_stride_b > (int64_t)1 << 40)) return SVA_ERR_SHAPE;
  if (!aligned(freq, 8) || !aligned(positions, 4)) return SVA_ERR_ALIGNMENT;
  const size_t item = item_of(p->dtype);
  Tensor qi, qo, ki{}, ko{};
  int st;
  if ((st = check_heads(q_in, B, N, D, item, false, false, &qi)) != SVA_OK) return st;
  if ((st = check_heads(q_out, B, N, D, item, false, true, &qo)) != SVA_OK) return st;
  if (qi.v.heads != qo.v.heads) return SVA_ERR_SHAPE;
  const bool q_place = same(qi, qo, B, N);
  if (!q_place && !apart(qi, qo)) return SVA_ERR_INVALID_ARG;
  int piece = std::min(qi.align, qo.align);
  bool k_place = true;
  if (k_in) {
    if ((st = check_heads(k_in, B, N, D, item, false, false, &ki)) != SVA_OK) return st;
    if ((st = check_heads(k_out, B, N, D, item, false, true, &ko)) != SVA_OK) return st;
    if (ki.v.heads != ko.v.heads) return SVA_ERR_SHAPE;
    k_place = same(ki, ko, B, N);
    if (!k_place && !apart(ki, ko)) return SVA_ERR_INVALID_ARG;
    if (qo.v.p == ko.v.p || qo.v.p == ki.v.p || ko.v.p == qi.v.p) return SVA_ERR_INVALID_ARG;
    piece = std::min({piece, ki.align, ko.align});
  }
  if ((int64_t)qi.v.heads + ki.v.heads > 1 << 20) return SVA_ERR_SHAPE;
  sva::RotaryArgs a{};
  a.qi = qi.v;
  a.qo = qo.v;
  a.ki = ki.v;
  a.ko = ko.v;
  a.freq = freq;
  a.pos = positions;
  a.pos_b = pos_stride_b;
  a.B = p->batch;
  a.N = p->tokens;
  a.D = p->head_dim;
  a.rot = p->rot_dim;
  a.magnitude = (float)p->magnitude;
  a.f32 = p->dtype == SVA_F32;
  a.half = p->layout == SVA_ROTARY_HALF;
  a.backward = p->backward != 0;
  a.copy = !(q_place && k_place);
  // bytes of an access: a whole number of them makes the turned part (each half of it) and the rest
  const int64_t turned = (int64_t)p->rot_dim * item / (a.half ? 2 : 1), row = a.copy ? D * (int64_t)item : 0;
  while (piece > (int)item && (turned % piece != 0 || row % piece != 0)) piece /= 2;
  a.piece = piece;
  const int64_t rest = a.copy ? (D - p->rot_dim) * (int64_t)item : 0;
  a.ragged = piece >= 4 && turned >= 16 && (rest == 0 || rest >= 16);
  return hip_status(sva::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

int sva_cache_write(const sva_cache* cache, int32_t batch, int32_t tokens, int32_t dtype, const sva_heads* k,
                    const sva_heads* v, const int32_t* slots, int64_t slots_stride_b, void* stream) {
  sva::CacheRowsArgs a{};
  const int st = check_rows(cache, batch, tokens, dtype, slots, slots_stride_b, k, v, false, &a);
  if (st != SVA_OK) return st;
  return hip_status(sva::launch_cache_write(a, static_cast<hipStream_t>(stream)));
}

int sva_cache_read(const sva_cache* cache, int32_t batch, int32_t tokens, int32_t dtype, const int32_t* slots,
                   int64_t slots_stride_b, const sva_heads* k, const sva_heads* v, void* stream) {
  sva::CacheRowsArgs a{};
  const int st = check_rows(cache, batch, tokens, dtype, slots, slots_stride_b, k, v, true, &a);
  if (st != SVA_OK) return st;
  return hip_status(sva::launch_cache_read(a, static_cast<hipStream_t>(stream)));
}

int sva_cache_attention_workspace(const sva_cache* cache, const sva_cache_query* query, size_t* bytes) {
  if (!bytes) return SVA_ERR_INVALID_ARG;
  sva::CacheAttnArgs a{};
  const int st = check_query(cache, false, query, &a);
  if (st != SVA_OK) return st;
  *bytes = sva::cache_attn_shape(a).ws_bytes;
  return SVA_OK;
}

int sva_cache_attention(const sva_cache* cache, const sva_cache_query* query, const sva_heads* q,
                        const int32_t* page_table, const int32_t* lengths, const sva_heads* k_new,
                        const sva_heads* v_new, const uint8_t* mask, int64_t mask_stride_b, const int32_t* counts,
                        void* workspace, size_t workspace_bytes, const sva_heads* out, float* lse, void* stream) {
  sva::CacheAttnArgs a{};
  int st = check_query(cache, true, query, &a);
  if (st != SVA_OK) return st;
  if (!page_table || !lengths || (!k_new) != (!v_new) || mask_stride_b < 0) return SVA_ERR_INVALID_ARG;
  if (mask && query->batch > 1 && mask_stride_b > (int64_t)1 << 40) return SVA_ERR_SHAPE;
  const int64_t B = a.B, T = a.T, D = cache->head_dim;
  const size_t item = item_of(query->out_dtype);
  Tensor tq, to, tk{}, tv{};
  if ((st = check_heads(q, B, T, D, 2, true, false, &tq)) != SVA_OK) return st;
  if ((st = check_heads(out, B, T, D, item, true, true, &to)) != SVA_OK) return st;
  if (tq.v.heads != a.H || to.v.heads != a.H) return SVA_ERR_SHAPE;
  if (k_new) {
    if ((st = check_heads(k_new, B, T, D, 2, true, false, &tk)) != SVA_OK) return st;
    if ((st = check_heads(v_new, B, T, D, 2, true, false, &tv)) != SVA_OK) return st;
    if (tk.v.heads != cache->kv_heads || tv.v.heads != cache->kv_heads) return SVA_ERR_SHAPE;
  }
  // outputs are written while other workgroups still read the inputs
  if (tq.v.p == to.v.p || (k_new && (tk.v.p == to.v.p || tv.v.p == to.v.p))) return SVA_ERR_INVALID_ARG;
  if (!aligned(page_table, 4) || !aligned(lengths, 4) || (counts && !aligned(counts, 4)) || (lse && !aligned(lse, 4)))
    return SVA_ERR_ALIGNMENT;
  const size_t need = sva::cache_attn_shape(a).ws_bytes;
  if (need > 0) {
    if (!workspace) return SVA_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SVA_ERR_SHAPE;
    if (!aligned(workspace, 256)) return SVA_ERR_ALIGNMENT;
  }
  a.q = tq.v;
  a.kn = tk.v;
  a.vn = tv.v;
  a.out = to.v;
  a.table = page_table;
  a.lens = lengths;
  a.mask = mask;
  a.mask_b = mask_stride_b;
  a.counts = counts;
  a.ws = static_cast<float*>(workspace);
  a.lse = lse;
  return hip_status(sva::launch_cache_attention(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
