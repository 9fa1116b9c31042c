// Attention of the newest tokens of every request over its cached tokens.
//
// The rows of a kv head are taken 16 or 32 at a time here (cache_rows.h), 64 or 32 in
// cache_tiles.h where there are more.
//
// Work is split along the pages where there are few rows: with W the pages of
// all tiles, a tile of n pages goes to ceil(n / X) workgroups, X just above W / A,
// A 512 less a share of the long tiles, 256 at least, and X not below the least
// pages of a part (64 or 128 KiB, twice that from 256 tiles on), so that a long
// request among short ones does not hold up the call.  The lengths are on the device; each wave forms the sums over
// the requests for itself.  Parts leave their sums and maxima in the workspace,
// and a second launch joins them, in the order of the pages.
#include "cache_rows.h"

namespace ugbs {
namespace {

template <int D, int DT, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) cache_attend_rows_kernel(CacheAttendParams P) {
  constexpr int ROWS = 16 * RT;
  __shared__ RowsMemory<D, RT, NW> memory;
  Part u;
  if (!find_part<ROWS, kParts>(P, blockIdx.x, &u)) return;
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.kvh = __builtin_amdgcn_readfirstlane(u.kvh);
  u.kv = __builtin_amdgcn_readfirstlane(u.kv);
  const int n = pages_seen<ROWS>(P, u);
  const int p0 = __builtin_amdgcn_readfirstlane(n * u.split / u.splits);
  const int p1 = __builtin_amdgcn_readfirstlane(n * (u.split + 1) / u.splits);
  rows_part<D, DT, RT, NW, kWhole>(P, u, u.splits > 1 ? ((int64_t)u.slot + u.split) * ROWS : -1, p0, p1, memory);
}

template <int D, int DT, int RT>
hipError_t attend_rows(const CacheAttendParams& P, hipStream_t stream) {
  constexpr int NW = 4, ROWS = 16 * RT;
  const int64_t units = tiles_bound(P.s, ROWS);
  launch_schedule<ROWS>(P, stream);
  cache_attend_rows_kernel<D, DT, RT, NW><<<(unsigned)(units + (P.splits ? kTarget : 0)), 64 * NW, 0, stream>>>(P);
  if (P.splits) launch_join<D, ROWS>(P, stream);
  return hipGetLastError();
}

// At d 256 32 rows leave one wave per SIMD here, two in cache_tiles.hip (8 requests of
// up to 30K, 4 rows of 8 heads, int8: 50 / 43 us).
template <int D, int DT>
hipError_t attend(const CacheAttendParams& P, hipStream_t stream) {
  const int64_t rows = (int64_t)P.s.rows * P.s.G;
  if (rows <= 16) return attend_rows<D, DT, 1>(P, stream);
  if constexpr (D != 256)
    if (rows <= 32) return attend_rows<D, DT, 2>(P, stream);
  return launch_cache_tiles(P, stream);
}

}  // namespace

// Workspace: the parts' sums, their (maximum, sum) pairs, and a large batch's schedule.
static size_t schedule_at(const CacheShape& s) {
  return may_split(s) ? (size_t)kSlots * tile_rows(s) * (s.d * sizeof(float) + sizeof(float2)) : 0;
}

size_t cache_attend_workspace(const CacheShape& s) {
  size_t n = schedule_at(s);
  if (s.B > kWaveBatch)
    n = align256(n) + align256(s.B * sizeof(int4)) + align256(schedule_entries(s, tile_rows(s)) * sizeof(int32_t)) +
        kTarget * sizeof(int32_t) + kLongTiles * sizeof(int2);
  return n;
}

hipError_t launch_cache_attend(const CacheShape& s, const uint16_t* Q, const uint8_t* cache, const float* scales,
                               const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens, uint16_t* O,
                               void* workspace, hipStream_t stream) {
  CacheAttendParams P{s, Q, cache, scales, table, kv_lens, q_lens, O, nullptr, nullptr, 0.f, false, {}, min_pages(s.d), {}};
  P.scale_log2 = s.scale * 1.4426950408889634f;
  P.splits = may_split(s);
  if (P.splits) {
    P.part_o = static_cast<float*>(workspace);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)kSlots * tile_rows(s) * s.d);
  }
  if (s.B > kWaveBatch) {
    uint8_t* const at = static_cast<uint8_t*>(workspace) + align256(schedule_at(s));
    P.schedule.request = reinterpret_cast<int4*>(at);
    P.schedule.part = reinterpret_cast<int32_t*>(at + align256(s.B * sizeof(int4)));
    P.schedule.join = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(P.schedule.part) +
                                                 align256(schedule_entries(s, tile_rows(s)) * sizeof(int32_t)));
    P.schedule.long_tile = reinterpret_cast<int2*>(P.schedule.join + kTarget);
  }
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) return f8 ? attend<64, UGBS_E4M3>(P, stream) : attend<64, UGBS_INT8>(P, stream);
  if (s.d == 128) return f8 ? attend<128, UGBS_E4M3>(P, stream) : attend<128, UGBS_INT8>(P, stream);
  return f8 ? attend<256, UGBS_E4M3>(P, stream) : attend<256, UGBS_INT8>(P, stream);
}

}  // namespace ugbs
