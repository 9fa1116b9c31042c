// The 8-bit key/value cache: its layout in memory, the conversions between its
// bytes and bf16, and the launchers of its kernels.
//
// A page holds 64 tokens.  Page p of kv head h is 64 d bytes of keys, then
// 64 d bytes of values.  Both are kept in the order in which the attention's
// matrix instructions take them, 16 bytes per lane, so a wave's loads are
// 1 KiB in a row and need no shared memory to be rearranged:
//   keys    [t / 16][c / 64][c % 64 / 16][t % 16][c % 16]: one load is a
//           16-token tile, lane (group g, token t) holding 16 channels: the A
//           operands (8 channels each) of two steps along d;
//   values  [t / 32][c / 32][t % 16 / 4][c % 16][c % 32 / 16][t % 32 / 16][t % 4]:
//           one load is 32 tokens of 32 channels, lane (group g, channel c)
//           holding two A operands of V^T: 8 tokens of channels c and c + 16,
//           in the order in which a lane holds its probabilities.
#pragma once
#include "attend_common.h"

namespace ugbs {

struct CacheShape {
  int B, H, Hkv, G, d, n_pages, max_pages, rows, dtype;
  float scale;
};

hipError_t launch_cache_plan(const CacheShape& s, const int32_t* ctx_lens, const int32_t* new_lens, int32_t* free_pages,
                             const int32_t* free_count, int32_t* table, int32_t* kv_lens, int32_t* q_lens, int32_t* slots,
                             int32_t* free_left, hipStream_t stream);
hipError_t launch_cache_store(const CacheShape& s, const uint16_t* K, const uint16_t* V, const int32_t* slots, uint8_t* cache,
                              float* scales, hipStream_t stream);
hipError_t launch_cache_load(const CacheShape& s, const uint8_t* cache, const float* scales, const int32_t* table,
                             const int32_t* start, const int32_t* count, int width, uint16_t* K, uint16_t* V,
                             hipStream_t stream);
hipError_t launch_cache_attend(const CacheShape& s, const uint16_t* Q, const uint8_t* cache, const float* scales,
                               const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens, uint16_t* O,
                               void* workspace, hipStream_t stream);
size_t cache_attend_workspace(const CacheShape& s);

namespace {

// Position of (token t, channel c) within the keys or the values of a page.
template <int D>
__host__ __device__ constexpr int key_at(int t, int c) {
  return (t >> 4) * 16 * D + (c >> 6) * 1024 + ((c >> 4) & 3) * 256 + (t & 15) * 16 + (c & 15);
}
template <int D>
__host__ __device__ constexpr int value_at(int t, int c) {
  return (t >> 5) * 32 * D + (c >> 5) * 1024 + ((t >> 2) & 3) * 256 + (c & 15) * 16 + ((c >> 4) & 1) * 8 + ((t >> 4) & 1) * 4 + (t & 3);
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp(int x) {      // 0 where the lane has no source
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROW_MASK, 0xf, false);
}

// Sum over lanes 0 .. l (shifts within 16 lanes, then the last lane of a row to the next rows).
__device__ __forceinline__ int scan_add(int x) {
  x += dpp<0x111, 0xf>(x);
  x += dpp<0x112, 0xf>(x);
  x += dpp<0x114, 0xf>(x);
  x += dpp<0x118, 0xf>(x);
  x += dpp<0x142, 0xa>(x);
  x += dpp<0x143, 0xc>(x);
  return x;
}

// x, opaque to the compiler: what follows from it is formed where it is used, not kept
// in registers over a loop or from before a rare branch.
__device__ __forceinline__ uint32_t here(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// 16 bytes that are read once: not kept in the caches (a decode step over 300 MB:
// 64 -> 57 us).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// Four bytes of the cache as four bf16 (exact: e4m3 has 4 significant bits and
// the integers 7).  e4m3: times a scale, a power of two, which the conversion takes
// along; integers: the scale is applied elsewhere.
template <int DT>
__device__ __forceinline__ uint2 bytes_to_bf16(uint32_t w, float scale) {
  if constexpr (DT == UGBS_E4M3) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)));
  } else {
    const float a = (float)(int8_t)w, b = (float)(int8_t)(w >> 8), c = (float)(int8_t)(w >> 16), d = (float)(int8_t)(w >> 24);
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u),
                      __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x07060302u));
  }
}

// Eight bytes as the A operand of a matrix instruction.
template <int DT>
__device__ __forceinline__ bf16x8 operand(uint32_t lo, uint32_t hi, float scale = 1.0f) {
  const uint2 a = bytes_to_bf16<DT>(lo, scale), b = bytes_to_bf16<DT>(hi, scale);
  return as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
}

}  // namespace
}  // namespace ugbs
