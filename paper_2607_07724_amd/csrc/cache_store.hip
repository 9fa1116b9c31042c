// Keys and values by heads into the cache's pages (8 bits, one scale per page
// and kv head for each; cache_store.h), and back out as bf16.
#include "cache_store.h"

namespace ugbs {
namespace {

// Keys and values by heads: a thread has the same 4 tokens and 8 channels of both.
template <int D>
struct HeadRows {
  static constexpr bool kSameTokens = true;
  const uint16_t* K;
  const uint16_t* V;
  int Hkv, rows;
  __device__ __forceinline__ int key_token(int e) const { return (int)threadIdx.x / (D / 8) * 4 + e; }
  __device__ __forceinline__ int key_channel(int) const { return (int)threadIdx.x % (D / 8) * 8; }
  __device__ __forceinline__ void load(int b, int kvh, int at, int, int, uint32_t, uint32_t live, uint4 (&k)[4], uint4 (&v)[4]) const {
    const size_t base = ((size_t)b * Hkv + kvh) * rows;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = v[e] = make_uint4(0, 0, 0, 0);
      if (live >> e & 1) {
        const size_t from = (base + at + key_token(e)) * D + key_channel(e);
        k[e] = *reinterpret_cast<const uint4*>(K + from);
        v[e] = *reinterpret_cast<const uint4*>(V + from);
      }
    }
  }
};

template <int D, int DT>
__global__ void __launch_bounds__(2 * D) cache_store_kernel(CacheShape s, const uint16_t* __restrict__ K,
                                                            const uint16_t* __restrict__ V,
                                                            const int32_t* __restrict__ slots, uint8_t* __restrict__ cache,
                                                            float* __restrict__ scales, int pages_each) {
  __shared__ __align__(16) uint8_t s_page[2][kBlock * D];
  store_page<D, DT>(s, HeadRows<D>{K, V, s.Hkv, s.rows}, slots, cache, scales, pages_each, blockIdx.x, s_page);
}

// Cached tokens as bf16.  One workgroup per (request, kv head, page of the
// window): the page is read 16 bytes a lane into LDS, and leaves it as rows.
template <int D, int DT>
__global__ void __launch_bounds__(2 * D) cache_load_kernel(CacheShape s, const uint8_t* __restrict__ cache,
                                                           const float* __restrict__ scales,
                                                           const int32_t* __restrict__ table,
                                                           const int32_t* __restrict__ start,
                                                           const int32_t* __restrict__ count, int width,
                                                           uint16_t* __restrict__ K, uint16_t* __restrict__ V,
                                                           int pages_each) {
  constexpr int CG = D / 8;
  __shared__ __align__(16) uint8_t s_page[2][kBlock * D];
  const int tid = threadIdx.x;
  int u = blockIdx.x;
  const int kvh = u % s.Hkv;
  u /= s.Hkv;
  const int j = u % pages_each, b = u / pages_each;
  const int n = min(max(count[b], 0), width);
  const int from = min(max(start[b], 0), s.max_pages * kBlock);
  const int p = from / kBlock + j;          // the window's j-th page
  const int i0 = p * kBlock - from;         // its first token's row
  if (i0 >= n) return;
  const int page = p < s.max_pages ? table[(size_t)b * s.max_pages + p] : -1;
  const bool there = page >= 0 && page < s.n_pages;
  float ks = 0.f, vs = 0.f;
  if (there) {
    const float* const sc = scales + 2 * ((size_t)page * s.Hkv + kvh);
    ks = sc[0];
    vs = sc[1];
    const uint4* const src = reinterpret_cast<const uint4*>(cache + ((size_t)page * s.Hkv + kvh) * 2 * (kBlock * D));
#pragma unroll
    for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(s_page)[e * 2 * D + tid] = load_once(src + e * 2 * D + tid);
  }
  __syncthreads();
  const int cg = tid % CG, tg = tid / CG, c0 = 8 * cg;
  const size_t base = ((size_t)b * s.Hkv + kvh) * width;
  uint32_t vb[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) vb[c] = *reinterpret_cast<const uint32_t*>(s_page[1] + value_at<D>(4 * tg, c0 + c));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = i0 + 4 * tg + e;
    if (i < 0 || i >= n) continue;
    uint4 ko = make_uint4(0, 0, 0, 0), vo = ko;
    if (there) {
      const uint2 kb = *reinterpret_cast<const uint2*>(s_page[0] + key_at<D>(4 * tg + e, c0));
      uint32_t kk[4], vv[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t w = c < 2 ? kb.x : kb.y;
        kk[c] = pack_bf16(number_of<DT>(w, 2 * (c & 1)) * ks, number_of<DT>(w, 2 * (c & 1) + 1) * ks);
        vv[c] = pack_bf16(number_of<DT>(vb[2 * c], e) * vs, number_of<DT>(vb[2 * c + 1], e) * vs);
      }
      ko = make_uint4(kk[0], kk[1], kk[2], kk[3]);
      vo = make_uint4(vv[0], vv[1], vv[2], vv[3]);
    }
    *reinterpret_cast<uint4*>(K + (base + i) * D + c0) = ko;
    *reinterpret_cast<uint4*>(V + (base + i) * D + c0) = vo;
  }
}

template <int D, int DT>
void store(const CacheShape& s, const uint16_t* K, const uint16_t* V, const int32_t* slots, uint8_t* cache, float* scales,
           hipStream_t stream) {
  const int each = pages_touched(s.rows);
  cache_store_kernel<D, DT><<<(unsigned)((int64_t)s.B * s.Hkv * each), 2 * D, 0, stream>>>(s, K, V, slots, cache, scales, each);
}

template <int D, int DT>
void load(const CacheShape& s, const uint8_t* cache, const float* scales, const int32_t* table, const int32_t* start,
          const int32_t* count, int width, uint16_t* K, uint16_t* V, hipStream_t stream) {
  const int each = pages_touched(width);
  cache_load_kernel<D, DT><<<(unsigned)((int64_t)s.B * s.Hkv * each), 2 * D, 0, stream>>>(s, cache, scales, table, start, count,
                                                                                      width, K, V, each);
}

}  // namespace

hipError_t launch_cache_store(const CacheShape& s, const uint16_t* K, const uint16_t* V, const int32_t* slots, uint8_t* cache,
                              float* scales, hipStream_t stream) {
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) (f8 ? store<64, UGBS_E4M3> : store<64, UGBS_INT8>)(s, K, V, slots, cache, scales, stream);
  else if (s.d == 128) (f8 ? store<128, UGBS_E4M3> : store<128, UGBS_INT8>)(s, K, V, slots, cache, scales, stream);
  else (f8 ? store<256, UGBS_E4M3> : store<256, UGBS_INT8>)(s, K, V, slots, cache, scales, stream);
  return hipGetLastError();
}

hipError_t launch_cache_load(const CacheShape& s, const uint8_t* cache, const float* scales, const int32_t* table,
                             const int32_t* start, const int32_t* count, int width, uint16_t* K, uint16_t* V,
                             hipStream_t stream) {
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) (f8 ? load<64, UGBS_E4M3> : load<64, UGBS_INT8>)(s, cache, scales, table, start, count, width, K, V, stream);
  else if (s.d == 128) (f8 ? load<128, UGBS_E4M3> : load<128, UGBS_INT8>)(s, cache, scales, table, start, count, width, K, V, stream);
  else (f8 ? load<256, UGBS_E4M3> : load<256, UGBS_INT8>)(s, cache, scales, table, start, count, width, K, V, stream);
  return hipGetLastError();
}

}  // namespace ugbs
