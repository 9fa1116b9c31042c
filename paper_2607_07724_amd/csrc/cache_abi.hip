// extern "C" boundary of the cache's entry points: argument validation, derived
// sizes and dispatch.  Every check runs before anything is enqueued; nothing here
// allocates, frees or synchronises.
#include "cache_check.h"

namespace {

using ugbs::CacheShape;
using ugbs::make_cache;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? UGBS_OK : UGBS_ERR_HIP; }

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
  if (width < 1 || width > UGBS_MAX_WIDTH || !ugbs::grid_fits((int64_t)s.B * s.Hkv, width)) return UGBS_ERR_SHAPE;
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

size_t ugbs_cache_share_bytes(const ugbs_cache* c) {
  CacheShape s;
  return make_cache(c, &s) == UGBS_OK ? ugbs::cache_share_bytes(s) : 0;
}

size_t ugbs_cache_shared_workspace_bytes(const ugbs_cache* c) {
  CacheShape s;
  return make_cache(c, &s) == UGBS_OK ? ugbs::cache_shared_workspace(s) : 0;
}

int ugbs_cache_share(const ugbs_cache* c, const int32_t* group, const int32_t* table, const int32_t* kv_lens,
                     const int32_t* q_lens, void* share, size_t share_bytes, void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  if (!group || !table || !kv_lens || !q_lens) return UGBS_ERR_NULL;
  if (!share || share_bytes < ugbs::cache_share_bytes(s)) return UGBS_ERR_WORKSPACE;
  if (!aligned(group, 4) || !aligned(table, 4) || !aligned(kv_lens, 4) || !aligned(q_lens, 4) || !aligned(share, 256))
    return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_cache_share(s, group, table, kv_lens, q_lens, share, static_cast<hipStream_t>(stream)));
}

int ugbs_cache_attend_shared(const ugbs_cache* c, const void* Q, const void* cache, const float* scales, const int32_t* table,
                             const int32_t* kv_lens, const int32_t* q_lens, const void* share, size_t share_bytes, void* O,
                             void* workspace, size_t workspace_bytes, void* stream) {
  CacheShape s;
  const int st = make_cache(c, &s);
  if (st) return st;
  if (!Q || !cache || !scales || !table || !kv_lens || !q_lens || !O) return UGBS_ERR_NULL;
  const size_t need = ugbs::cache_shared_workspace(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return UGBS_ERR_WORKSPACE;
  if (!share || share_bytes < ugbs::cache_share_bytes(s)) return UGBS_ERR_WORKSPACE;
  if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(cache, 16) || !aligned(scales, 8) || !aligned(table, 4) ||
      !aligned(kv_lens, 4) || !aligned(q_lens, 4) || !aligned(share, 256) || (need > 0 && !aligned(workspace, 256)))
    return UGBS_ERR_ALIGN;
  return hip_status(ugbs::launch_cache_attend_shared(s, static_cast<const uint16_t*>(Q), static_cast<const uint8_t*>(cache),
                                                     scales, table, kv_lens, q_lens, share, static_cast<uint16_t*>(O), workspace,
                                                     static_cast<hipStream_t>(stream)));
}

}  // extern "C"
