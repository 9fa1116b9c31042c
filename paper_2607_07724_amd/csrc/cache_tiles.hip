// Attention over the cache where a request brings many rows (pieces of prompts): cache_tiles.h.
#include "cache_tiles.h"

namespace ugbs {
namespace {

template <int D, int DT, int RT, int QR, int NW, int WPE, bool ONCE>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
cache_tiles_kernel(CacheAttendParams P) {
  constexpr int ROWS = 16 * RT;
  __shared__ TilesMemory<D, DT, RT, QR, NW> memory;
  Part u;
  if (!find_part<ROWS, kGroups>(P, blockIdx.x, &u)) return;
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.kvh = __builtin_amdgcn_readfirstlane(u.kvh);
  u.kv = __builtin_amdgcn_readfirstlane(u.kv);
  u.q = __builtin_amdgcn_readfirstlane(u.q);
  u.tile = __builtin_amdgcn_readfirstlane(u.tile);
  const int n = pages_seen<ROWS>(P, u);
  const int p0 = __builtin_amdgcn_readfirstlane(n * u.split / u.splits);
  const int p1 = __builtin_amdgcn_readfirstlane(n * (u.split + 1) / u.splits);
  tiles_part<D, DT, RT, QR, NW, ONCE, kWhole>(P, u, u.splits > 1 ? ((int64_t)u.slot + u.split) * ROWS : -1, p0, p1, memory);
}

template <int D, int DT, int RT, int QR, int WPE>
hipError_t tiles(const CacheAttendParams& P, hipStream_t stream) {
  constexpr int NW = 4, ROWS = 16 * RT;
  static_assert(ROWS == tile_rows_many(D), "rows of a tile");
  const int64_t units = tiles_bound(P.s, ROWS);
  launch_schedule<ROWS>(P, stream);
  const unsigned grid = (unsigned)(units + (P.splits ? kTarget : 0));
  if ((int64_t)P.s.rows * P.s.G <= ROWS) cache_tiles_kernel<D, DT, RT, QR, NW, WPE, true><<<grid, 64 * NW, 0, stream>>>(P);
  else cache_tiles_kernel<D, DT, RT, QR, NW, WPE, false><<<grid, 64 * NW, 0, stream>>>(P);
  if (P.splits) launch_join<D, ROWS>(P, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_tiles(const CacheAttendParams& P, hipStream_t stream) {
  const bool f8 = P.s.dtype == UGBS_E4M3;
  if (P.s.d == 64) return f8 ? tiles<64, UGBS_E4M3, 4, 4, 3>(P, stream) : tiles<64, UGBS_INT8, 4, 4, 3>(P, stream);
  if (P.s.d == 128) return f8 ? tiles<128, UGBS_E4M3, 4, 2, 2>(P, stream) : tiles<128, UGBS_INT8, 4, 2, 2>(P, stream);
  return f8 ? tiles<256, UGBS_E4M3, 2, 2, 2>(P, stream) : tiles<256, UGBS_INT8, 2, 2, 2>(P, stream);
}

}  // namespace ugbs
