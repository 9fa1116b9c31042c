// What a cache's description has to satisfy (host code of the entry points).
#pragma once
#include <cmath>

#include "cache_internal.h"

namespace ugbs {
namespace {

// Workgroups that touch n consecutive tokens' pages, of up to 512 threads: a grid holds 2^32 threads.
inline bool grid_fits(int64_t batch_heads, int64_t n) { return batch_heads * ((n + 62) / 64 + 1) <= (1 << 22); }

inline int make_cache(const ugbs_cache* c, CacheShape* s) {
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
}  // namespace ugbs
