// extern "C" boundary of the entry points from a projection's rows to heads: argument
// validation and dispatch.  Every check runs before anything is enqueued; nothing here
// allocates, frees or synchronises.
#include "cache_check.h"
#include "heads_internal.h"

namespace {

using ugbs::CacheShape;
using ugbs::HeadsParams;
using ugbs::HeadsShape;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? UGBS_OK : UGBS_ERR_HIP; }

int make_heads(const ugbs_heads* h, HeadsShape* s) {
  if (!h) return UGBS_ERR_NULL;
  if (h->batch < 1 || h->batch > UGBS_MAX_REQUESTS) return UGBS_ERR_SHAPE;
  if (h->n_heads < 1 || h->n_kv_heads < 1 || h->n_heads % h->n_kv_heads) return UGBS_ERR_SHAPE;
  if ((int64_t)h->n_heads + 2 * (int64_t)h->n_kv_heads > 4096) return UGBS_ERR_SHAPE;
  if (h->head_dim != 64 && h->head_dim != 128 && h->head_dim != 256) return UGBS_ERR_SHAPE;
  if (h->rows < 1 || (int64_t)h->batch * h->rows > UGBS_MAX_TOKENS) return UGBS_ERR_SHAPE;
  if (h->rot_dim < 0 || h->rot_dim > h->head_dim || h->rot_dim % 16) return UGBS_ERR_ROTARY;
  if (h->pairs != UGBS_HALVES && h->pairs != UGBS_NEIGHBOURS) return UGBS_ERR_ROTARY;
  if (h->axes < 1 || h->axes > UGBS_MAX_AXES) return UGBS_ERR_ROTARY;
  if (!std::isfinite(h->norm_eps) || h->norm_eps < 0.0f || !std::isfinite(h->rot_gain)) return UGBS_ERR_ROTARY;
  *s = HeadsShape{h->batch, h->n_heads, h->n_kv_heads, h->head_dim, h->rows, h->rot_dim, h->pairs, h->axes, h->norm_eps,
                  h->rot_gain != 0.0f ? h->rot_gain : 1.0f};
  return UGBS_OK;
}

// What both entry points read, and the queries.
int make_params(const ugbs_heads* h, const ugbs_rows* q, const ugbs_rows* k, const ugbs_rows* v, const float* q_norm,
                const float* k_norm, const double* freqs, const int32_t* positions, const int32_t* axis, const int32_t* first,
                const int32_t* lens, void* Q, HeadsParams* P) {
  const int st = make_heads(h, &P->s);
  if (st) return st;
  for (const ugbs_rows* r : {q, k, v})
    if (!r || !r->at) return UGBS_ERR_NULL;
  if (!Q || (P->s.rot > 0 && !freqs)) return UGBS_ERR_NULL;
  for (const ugbs_rows* r : {q, k, v})
    if (r->batch % 8 || r->token % 8 || r->head % 8) return UGBS_ERR_STRIDE;
  for (const void* p : {q->at, k->at, v->at, static_cast<const void*>(q_norm), static_cast<const void*>(k_norm), static_cast<const void*>(Q)})
    if (!aligned(p, 16)) return UGBS_ERR_ALIGN;
  if (!aligned(freqs, 8)) return UGBS_ERR_ALIGN;
  for (const int32_t* p : {positions, axis, first, lens})
    if (!aligned(p, 4)) return UGBS_ERR_ALIGN;
  P->q = *q;
  P->k = *k;
  P->v = *v;
  P->q_norm = q_norm;
  P->k_norm = k_norm;
  P->freqs = freqs;
  P->axis = axis;
  P->positions = positions;
  P->first = first;
  P->lens = lens;
  P->Q = static_cast<uint16_t*>(Q);
  P->K = P->V = nullptr;
  return UGBS_OK;
}

}  // namespace

extern "C" {

int ugbs_heads_split(const ugbs_heads* h, const ugbs_rows* q, const ugbs_rows* k, const ugbs_rows* v, const float* q_norm,
                     const float* k_norm, const double* freqs, const int32_t* positions, const int32_t* axis,
                     const int32_t* first, const int32_t* lens, void* Q, void* K, void* V, void* stream) {
  HeadsParams P;
  const int st = make_params(h, q, k, v, q_norm, k_norm, freqs, positions, axis, first, lens, Q, &P);
  if (st) return st;
  if (!K || !V) return UGBS_ERR_NULL;
  if (!aligned(K, 16) || !aligned(V, 16)) return UGBS_ERR_ALIGN;
  P.K = static_cast<uint16_t*>(K);
  P.V = static_cast<uint16_t*>(V);
  return hip_status(ugbs::launch_heads_split(P, static_cast<hipStream_t>(stream)));
}

int ugbs_heads_store(const ugbs_heads* h, const ugbs_cache* c, const ugbs_rows* q, const ugbs_rows* k, const ugbs_rows* v,
                     const float* q_norm, const float* k_norm, const double* freqs, const int32_t* positions,
                     const int32_t* axis, const int32_t* first, const int32_t* lens, void* Q, const int32_t* slots, void* cache,
                     float* scales, void* stream) {
  HeadsParams P;
  const int st = make_params(h, q, k, v, q_norm, k_norm, freqs, positions, axis, first, lens, Q, &P);
  if (st) return st;
  CacheShape s;
  const int sc = ugbs::make_cache(c, &s);
  if (sc) return sc;
  if (s.B != P.s.B || s.H != P.s.H || s.Hkv != P.s.Hkv || s.d != P.s.d || s.rows != P.s.rows) return UGBS_ERR_SHAPE;
  if (!slots || !cache || !scales) return UGBS_ERR_NULL;
  if (!aligned(slots, 4) || !aligned(cache, 16) || !aligned(scales, 8)) return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_heads_store(P, s, slots, static_cast<uint8_t*>(cache), scales, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
