// Keys and values into the cache's pages (8 bits, one scale per page and kv
// head for each), and back out as bf16.
//
// A scale is the smallest power of two s >= 2^-100 with max |x| <= M s over
// the page's tokens, M the largest number of the type (448 or 127).  Why a
// power of two: x / s and the value read back are exact up to the one rounding
// to 8 bits; where a later token needs a larger scale, e4m3 bytes move to it
// without a second rounding (but for its subnormals), and the roundings of
// integers add up to less than one step, since every move at least halves them.
//
// One workgroup per (request, kv head, page that the call touches); a thread
// holds 4 consecutive tokens of 8 channels of both keys and values, so that
// the four tokens of a channel, which are adjacent in the values' layout, come
// out of one thread as a dword.  A whole page is put together in LDS and
// written 16 bytes a lane; in a page that held tokens before, or is not filled,
// bytes are written one token at a time and the others stay.
#include <type_traits>

#include "cache_internal.h"

namespace ugbs {
namespace {

constexpr float kTop[2] = {448.0f, 127.0f};

__device__ __forceinline__ float bf16_at(const uint4& v, int e) {
  const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
  return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
}

__device__ __forceinline__ uint32_t abs_max2(uint32_t m, uint32_t w) {
  const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
  return max(m, max(lo, hi));
}

// The same of numbers that are finite (a rare branch: see here()).
__device__ __forceinline__ uint32_t finite_max2(uint32_t m, uint32_t w) {
  w = here(w);
  const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
  return max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
}

// The scale of a page whose largest |x| has the bf16 pattern a.
template <int DT>
__device__ __forceinline__ float scale_for(uint32_t a) {
  const int x = (int)(a >> 7) - 127;
  const uint32_t m = a & 0x7f;
  // M is 1.75 2^8 (e4m3) or 1.984375 2^6 (int8)
  const int e = DT == UGBS_E4M3 ? x - 8 + (m > 0x60 ? 1 : 0) : x - 6 + (m > 0x7e ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}

// Four numbers (already divided by the scale) to bytes: nearest, ties to even.
template <int DT>
__device__ __forceinline__ uint32_t to_bytes(float a, float b, float c, float d) {
  constexpr float top = kTop[DT];
  a = fminf(fmaxf(a, -top), top);
  b = fminf(fmaxf(b, -top), top);
  c = fminf(fmaxf(c, -top), top);
  d = fminf(fmaxf(d, -top), top);
  if constexpr (DT == UGBS_E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    const uint32_t ia = (uint32_t)(int)rintf(a), ib = (uint32_t)(int)rintf(b), ic = (uint32_t)(int)rintf(c), id = (uint32_t)(int)rintf(d);
    return (ia & 0xff) | ((ib & 0xff) << 8) | ((ic & 0xff) << 16) | (id << 24);
  }
}

template <int DT>
__device__ __forceinline__ float number_of(uint32_t w, int byte) {
  if constexpr (DT == UGBS_E4M3) {
    switch (byte) {
      case 0: return __builtin_amdgcn_cvt_f32_fp8(w, 0);
      case 1: return __builtin_amdgcn_cvt_f32_fp8(w, 1);
      case 2: return __builtin_amdgcn_cvt_f32_fp8(w, 2);
      default: return __builtin_amdgcn_cvt_f32_fp8(w, 3);
    }
  } else {
    return (float)(int8_t)(w >> (8 * byte));
  }
}

// A dword's bytes moved to a scale 1 / ratio as large.
template <int DT>
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float ratio) {
  return to_bytes<DT>(number_of<DT>(w, 0) * ratio, number_of<DT>(w, 1) * ratio, number_of<DT>(w, 2) * ratio,
                      number_of<DT>(w, 3) * ratio);
}

template <int D, int DT>
__global__ void __launch_bounds__(2 * D) cache_store_kernel(CacheShape s, const uint16_t* __restrict__ K,
                                                            const uint16_t* __restrict__ V,
                                                            const int32_t* __restrict__ slots, uint8_t* __restrict__ cache,
                                                            float* __restrict__ scales, int pages_each) {
  constexpr int CG = D / 8;                 // threads along a row
  constexpr int NW = 2 * D / 64;
  __shared__ __align__(16) uint8_t s_page[2][kBlock * D];
  __shared__ uint32_t s_amax[NW][2];
  const int tid = threadIdx.x, w = tid >> 6;
  int u = blockIdx.x;
  const int kvh = u % s.Hkv;
  u /= s.Hkv;
  const int j = u % pages_each, b = u / pages_each;
  const int32_t* const slot = slots + (size_t)b * s.rows;
  // the first row's place in its page decides which rows belong to the j-th page touched
  const int s0 = slot[0];
  int i0 = 0, t0 = 0;
  if (s0 >= 0) {
    t0 = j == 0 ? s0 % kBlock : 0;
    i0 = max(0, j * kBlock - s0 % kBlock);
  } else {
    // no page for the first row: the j-th one begins at the row among 64 j - 63 .. 64 j that is its token 0
    if (j == 0) return;
    const int i = j * kBlock - (kBlock - 1) + (tid & 63), x = i < s.rows ? slot[i] : -1;
    const unsigned long long begins = __ballot(x >= 0 && x % kBlock == 0);
    if (!begins) return;
    i0 = j * kBlock - __builtin_clzll(begins);
  }
  if (i0 >= s.rows) return;
  const int i1 = min(s.rows, i0 + kBlock - t0);
  // this thread's 4 tokens and 8 channels; the slots of its rows come with the first one's
  const int cg = tid % CG, tg = tid / CG, c0 = 8 * cg;
  int mine[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) mine[e] = slot[min(max(i0 + 4 * tg + e - t0, i0), i1 - 1)];
  const int first = slot[i0];               // the page's first new token
  if (first < 0) return;
  const int page = first / kBlock;
  if (page >= s.n_pages || first % kBlock != t0) return;
  float* const sc = scales + 2 * ((size_t)page * s.Hkv + kvh);
  const float2 old = t0 > 0 ? *reinterpret_cast<const float2*>(sc) : make_float2(0.f, 0.f);
  uint4 k[4], v[4];
  uint32_t live = 0, ka = 0, va = 0;        // live: bit t of the thread's tokens that are new here
  const size_t base = ((size_t)b * s.Hkv + kvh) * s.rows;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int t = 4 * tg + e, i = i0 + t - t0;
    k[e] = v[e] = make_uint4(0, 0, 0, 0);
    // a row whose slot is not the next one of the page is left out
    if (i >= i0 && i < i1 && mine[e] == page * kBlock + t) {
      live |= 1u << e;
      k[e] = *reinterpret_cast<const uint4*>(K + (base + i) * D + c0);
      v[e] = *reinterpret_cast<const uint4*>(V + (base + i) * D + c0);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ka = abs_max2(abs_max2(abs_max2(abs_max2(ka, k[e].x), k[e].y), k[e].z), k[e].w);
    va = abs_max2(abs_max2(abs_max2(abs_max2(va, v[e].x), v[e].y), v[e].z), v[e].w);
  }
  int whole = 0;
  auto page_max = [&]() {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      ka = max(ka, (uint32_t)__shfl_xor((int)ka, o));
      va = max(va, (uint32_t)__shfl_xor((int)va, o));
    }
    if ((tid & 63) == 0) {
      s_amax[w][0] = ka;
      s_amax[w][1] = va;
    }
    whole = __syncthreads_and(live == 15u);
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      ka = max(ka, s_amax[x][0]);
      va = max(va, s_amax[x][1]);
    }
  };
  page_max();
  // a number that is not finite must not take the scale, and with it the page's other tokens, along
  const bool finite = __builtin_amdgcn_readfirstlane(max(ka, va)) < 0x7f80;
  if (!finite) {
    ka = va = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ka = finite_max2(finite_max2(finite_max2(finite_max2(ka, k[e].x), k[e].y), k[e].z), k[e].w);
      va = finite_max2(finite_max2(finite_max2(finite_max2(va, v[e].x), v[e].y), v[e].z), v[e].w);
    }
    __syncthreads();
    page_max();
  }
  float ks = scale_for<DT>(ka), vs = scale_for<DT>(va);
  uint8_t* const kp = cache + ((size_t)page * s.Hkv + kvh) * 2 * (kBlock * D);
  uint8_t* const vp = kp + kBlock * D;
  if (t0 > 0) {
    ks = fmaxf(ks, old.x);
    vs = fmaxf(vs, old.y);
    const float kr = old.x / ks, vr = old.y / vs;
    // tokens 0 .. t0 - 1 move to the larger scale
    if (kr < 1.0f) {
      for (int at = tid; at < kBlock * D / 16; at += 2 * D) {       // 16 channels of one token
        const int t = at / D * 16 + at % 16;
        if (t < t0) {
          uint4* const q = reinterpret_cast<uint4*>(kp) + at;
          const uint4 x = *q;
          *q = make_uint4(rescaled<DT>(x.x, kr), rescaled<DT>(x.y, kr), rescaled<DT>(x.z, kr), rescaled<DT>(x.w, kr));
        }
      }
    }
    if (vr < 1.0f) {
      for (int at = tid; at < kBlock * D / 4; at += 2 * D) {        // 4 tokens of one channel
        const int t = at / (8 * D) * 32 + (at & 1) * 16 + ((at >> 6) & 3) * 4;
        if (t < t0) {
          uint32_t* const q = reinterpret_cast<uint32_t*>(vp) + at;
          const uint32_t keep = t + 4 <= t0 ? 0u : ~0u << (8 * (t0 - t)), x = *q;
          *q = (rescaled<DT>(x, vr) & ~keep) | (x & keep);
        }
      }
    }
    __syncthreads();
  }
  // ---- to bytes: a scale is a power of two, so its reciprocal is exact
  const float ki = 1.0f / ks, vi = 1.0f / vs;
  uint2 kb[4];
  uint32_t vb[8];
  auto convert = [&](auto all_finite) {     // (else NaN become 0, infinities the largest number)
    auto at = [&](const uint4& from, int c, float inv) {
      if constexpr (all_finite.value) return bf16_at(from, c) * inv;
      const float x = bf16_at(make_uint4(here(from.x), here(from.y), here(from.z), here(from.w)), c) * inv;
      return x == x ? x : 0.f;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e)
      kb[e] = make_uint2(to_bytes<DT>(at(k[e], 0, ki), at(k[e], 1, ki), at(k[e], 2, ki), at(k[e], 3, ki)),
                         to_bytes<DT>(at(k[e], 4, ki), at(k[e], 5, ki), at(k[e], 6, ki), at(k[e], 7, ki)));
#pragma unroll
    for (int c = 0; c < 8; ++c) vb[c] = to_bytes<DT>(at(v[0], c, vi), at(v[1], c, vi), at(v[2], c, vi), at(v[3], c, vi));
  };
  if (finite) convert(std::true_type{});
  else convert(std::false_type{});

  if (whole) {
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<uint2*>(s_page[0] + key_at<D>(4 * tg + e, c0)) = kb[e];
#pragma unroll
    for (int c = 0; c < 8; ++c) *reinterpret_cast<uint32_t*>(s_page[1] + value_at<D>(4 * tg, c0 + c)) = vb[c];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
      reinterpret_cast<uint4*>(kp)[e * 2 * D + tid] = reinterpret_cast<const uint4*>(s_page)[e * 2 * D + tid];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (live >> e & 1) *reinterpret_cast<uint2*>(kp + key_at<D>(4 * tg + e, c0)) = kb[e];
    if (live == 15u) {
#pragma unroll
      for (int c = 0; c < 8; ++c) *reinterpret_cast<uint32_t*>(vp + value_at<D>(4 * tg, c0 + c)) = vb[c];
    } else if (live) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (live >> e & 1) {
#pragma unroll
          for (int c = 0; c < 8; ++c) vp[value_at<D>(4 * tg + e, c0 + c)] = (uint8_t)(vb[c] >> (8 * e));
        }
    }
  }
  if (tid == 0) *reinterpret_cast<float2*>(sc) = make_float2(ks, vs);
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

// Pages that n consecutive tokens can touch.
int pages_touched(int n) { return (n - 1 + kBlock - 1) / kBlock + 1; }

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
