// extern "C" boundary of the cache's entry points: argument validation, derived
// sizes and dispatch.  Every check runs before anything is enqueued; nothing here
// allocates, frees or synchronises.
#include <cmath>

#include "cache_internal.h"

namespace {

using ugbs::CacheShape;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? UGBS_OK : UGBS_ERR_HIP; }

// Workgroups that touch n consecutive tokens' pages, of up to 512 threads: a grid holds 2^32 threads.
bool grid_fits(int64_t batch_heads, int64_t n) { return batch_heads * ((n + 62) / 64 + 1) <= (1 << 22); }

int make_cache(const ugbs_cache* c, CacheShape* s) {
  if (!c) return UGBS_ERR_NULL;
  if (c->batch < 1 || c->batch > UGBS_MAX_REQUESTS) return UGBS_ERR_SHAPE;
  if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads) return UGBS_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return UGBS_ERR_SHAPE;
  if (c->n_pages < 1 || c->n_pages > UGBS_MAX_PAGES) return UGBS_ERR_SHAPE;
  if (c->max_pages < 1 || c->max_pages > UGBS_MAX_BLOCKS) return UGBS_ERR_SHAPE;
  if (c->rows < 1 || c->rows > c->max_pages * UGBS_BLOCK) return UGBS_ERR_SHAPE;
  if (c->dtype != UGBS_E4M3 && c->dtype != UGBS_INT8) return UGBS_ERR_DTYPE;
  if (!std::isfinite(c->softmax_scale) || c->softmax_scale < 0.0f) return UGBS_ERR_SCALE;
  const int G = c->n_heads / c->n_kv_heads;
  // grids of the kernels (tiles of 16 rows, 256 threads), and slots counted with 32 bits
  const int64_t heads = (int64_t)c->batch * c->n_kv_heads;
  if (heads > (1 << 22) || !grid_fits(heads, c->rows)) return UGBS_ERR_SHAPE;
  if ((int64_t)c->rows * G > (1 << 30) || heads * (((int64_t)c->rows * G + 15) / 16) > (1 << 23)) return UGBS_ERR_SHAPE;
  if ((int64_t)c->batch * c->rows > (1 << 30)) return UGBS_ERR_SHAPE;
  *s = CacheShape{c->batch, c->n_heads, c->n_kv_heads, G, c->head_dim, c->n_pages, c->max_pages, c->rows, c->dtype,
                  c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / std::sqrt((float)c->head_dim)};
  return UGBS_OK;
}

}  // namespace

extern "C" {

size_t ugbs_cache_workspace_bytes(const ugbs_cache* c) {
  CacheShape s;
  return make_cache(c, &s) == UGBS_OK ? ugbs::cache_attend_workspace(s) : 0;
}

int ugbs_cache_plan(const ugbs_cache* c, const int32_t* ctx_lens, const int32_t* new_lens, int32_t* free_pages,
                    const int32_t* free_count, int32_t* table, int32_t* kv_lens, int32_t* q_lens, int32_t* slots,
                    int32_t* free_left, void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  const void* const in[] = {ctx_lens, new_lens, free_pages, free_count, table};
  const void* const out[] = {kv_lens, q_lens, slots, free_left};
  for (const void* p : in)
    if (!p) return UGBS_ERR_NULL;
  for (const void* p : out)
    if (!p) return UGBS_ERR_NULL;
  for (const void* p : in)
    if (!aligned(p, 4)) return UGBS_ERR_ALIGN;
  for (const void* p : out)
    if (!aligned(p, 4)) return UGBS_ERR_ALIGN;
  for (int i = 0; i < 4; ++i) {
    for (const void* p : in)
      if (p == out[i]) return UGBS_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (out[j] == out[i]) return UGBS_ERR_ALIAS;
  }
  return hip_status(ugbs::launch_cache_plan(s, ctx_lens, new_lens, free_pages, free_count, table, kv_lens, q_lens, slots,
                                            free_left, static_cast<hipStream_t>(stream)));
}

int ugbs_cache_store(const ugbs_cache* c, const void* K, const void* V, const int32_t* slots, void* cache, float* scales,
                     void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  if (!K || !V || !slots || !cache || !scales) return UGBS_ERR_NULL;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 4) || !aligned(cache, 16) || !aligned(scales, 8))
    return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_cache_store(s, static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V), slots,
                                             static_cast<uint8_t*>(cache), scales, static_cast<hipStream_t>(stream)));
}

int ugbs_cache_load(const ugbs_cache* c, const void* cache, const float* scales, const int32_t* table, const int32_t* start,
                    const int32_t* count, int32_t width, void* K, void* V, void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  if (!cache || !scales || !table || !start || !count || !K || !V) return UGBS_ERR_NULL;
  if (width < 1 || width > UGBS_MAX_WIDTH || !grid_fits((int64_t)s.B * s.Hkv, width)) return UGBS_ERR_SHAPE;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(cache, 16) || !aligned(scales, 8) || !aligned(table, 4) ||
      !aligned(start, 4) || !aligned(count, 4))
    return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_cache_load(s, static_cast<const uint8_t*>(cache), scales, table, start, count, width,
                                            static_cast<uint16_t*>(K), static_cast<uint16_t*>(V),
                                            static_cast<hipStream_t>(stream)));
}

int ugbs_cache_attend(const ugbs_cache* c, const void* Q, const void* cache, const float* scales, const int32_t* table,
                      const int32_t* kv_lens, const int32_t* q_lens, void* O, void* workspace, size_t workspace_bytes,
                      void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  if (!Q || !cache || !scales || !table || !kv_lens || !q_lens || !O) return UGBS_ERR_NULL;
  const size_t need = ugbs::cache_attend_workspace(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return UGBS_ERR_WORKSPACE;
  if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(cache, 16) || !aligned(scales, 8) || !aligned(table, 4) ||
      !aligned(kv_lens, 4) || !aligned(q_lens, 4) || (need > 0 && !aligned(workspace, 256)))
    return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_cache_attend(s, static_cast<const uint16_t*>(Q), static_cast<const uint8_t*>(cache), scales,
                                              table, kv_lens, q_lens, static_cast<uint16_t*>(O), workspace,
                                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
