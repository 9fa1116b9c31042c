// A projection's rows as queries by heads, and as keys and values straight into the cache's
// pages: what heads.hip and cache_store.hip do one after the other, byte for byte, without
// the bf16 keys and values in between.  One launch: workgroups for the touched pages, and
// behind them those for the queries.
#include "cache_store.h"
#include "heads_internal.h"

namespace ugbs {
namespace {

// Keys and values of a page from a projection's rows.  Keys: d / 16 lanes to a row, as in
// split_heads, two rows (tokens t and t + 32) to a thread; their angles lie where the page is put
// together afterwards, those of 32 tokens at a time.
template <int D, int PAIRS>
struct ProjectionRows {
  static constexpr bool kSameTokens = false;
  static constexpr int LANES = D / 16;
  const HeadsParams& P;
  float2* s_angle;                          // [32][rot / 2]
  Angles<2 * D> angles;

  __device__ __forceinline__ int2 eights() const { return eights_of(P.s, (int)threadIdx.x % LANES); }
  __device__ __forceinline__ int key_token(int e) const { return (int)threadIdx.x / LANES + 32 * (e >> 1); }
  __device__ __forceinline__ int key_channel(int e) const { return e & 1 ? eights().y : eights().x; }

  __device__ __forceinline__ void load(int b, int kvh, int at, int t0, int t1, uint32_t live_k, uint32_t live_v, uint4 (&k)[4],
                                       uint4 (&v)[4]) const {
    const int tid = threadIdx.x, l = tid % LANES, half = P.s.rot / 2;
    const int2 c = eights();
    const uint16_t* const kr = row_at(P.k, b, 0, kvh);
    const uint16_t* const vr = row_at(P.v, b, 0, kvh) + tid % (D / 8) * 8;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = v[e] = make_uint4(0, 0, 0, 0);
      if (live_k >> e & 1) k[e] = *reinterpret_cast<const uint4*>(kr + (at + key_token(e)) * P.k.token + (e & 1 ? c.y : c.x));
      if (live_v >> e & 1) v[e] = *reinterpret_cast<const uint4*>(vr + (at + tid / (D / 8) * 4 + e) * P.v.token);
    }
    const bool turn = half > 0, rotated = 16 * l < P.s.rot;
    if (!turn && !P.k_norm) return;
    float wt[16];
    if (P.k_norm) weights_of(P.k_norm, c, wt);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int lo = max(t0, 32 * r), hi = min(t1, 32 * r + 32);
      if (lo >= hi) continue;
      float2 cs[8];
      if (turn) {
        if (r) __syncthreads();
        angles.fill(P, lo - 32 * r, hi - 32 * r, [&](int t) { return make_int2(b, at + 32 * r + t); }, s_angle);
        __syncthreads();
        angles_of<PAIRS>(P.s, s_angle + tid / LANES * half, l, cs);
      }
      if (P.k_norm) do_row<D, PAIRS, true>(k[2 * r], k[2 * r + 1], wt, cs, turn && rotated, P.s.eps);
      else do_row<D, PAIRS, false>(k[2 * r], k[2 * r + 1], wt, cs, rotated, P.s.eps);
      // places of a page that are not new hold angles of nothing
      if (!(live_k >> 2 * r & 1)) k[2 * r] = k[2 * r + 1] = make_uint4(0, 0, 0, 0);
    }
  }
};

template <int D, int DT, int PAIRS>
__global__ void __launch_bounds__(2 * D) heads_store_kernel(HeadsParams P, CacheShape c, const int32_t* __restrict__ slots,
                                                            uint8_t* __restrict__ cache, float* __restrict__ scales,
                                                            int pages_each, int stores, int groups, int heads_each) {
  __shared__ __align__(16) uint8_t s_page[2][kBlock * D];
  float2* const s_angle = reinterpret_cast<float2*>(&s_page[0][0]);
  // By eights (workgroup j runs on XCD j mod 8), one of pages, which wait for angles and maxima, to two of queries, which
  // wait for memory, while there are both.  (32K tokens of 28/4 heads: 115 us, pages first 123; 6 pieces of up to 777 tokens:
  // 17.0, pages first 16.6, pages spread over all 27.)
  const int e = blockIdx.x / 8, pages = (stores + 7) / 8, queries = gridDim.x / 8 - pages;
  auto pages_before = [&](int x) { return max(min((x + 2) / 3, pages), x - queries); };
  const int before = pages_before(e);
  if (pages_before(e + 1) > before) {
    const int u = 8 * before + blockIdx.x % 8;
    if (u < stores) store_page<D, DT>(c, ProjectionRows<D, PAIRS>{P, s_angle, Angles<2 * D>(P)}, slots, cache, scales, pages_each, u, s_page);
  } else {
    const int u = 8 * (e - before) + blockIdx.x % 8, h0 = u / groups * heads_each;
    if (h0 < P.s.H) split_heads<D, PAIRS, 2 * D / 64>(P, place_in_row(u % groups, groups) * kTokens<D>, h0, min(h0 + heads_each, P.s.H), s_angle);
  }
}

template <int D, int DT, int PAIRS>
void store(const HeadsParams& P, const CacheShape& c, const int32_t* slots, uint8_t* cache, float* scales, hipStream_t stream) {
  const int64_t groups = ((int64_t)P.s.B * P.s.rows + kTokens<D> - 1) / kTokens<D>;
  const int slices = head_slices(groups, P.s.H, 2 * D / 64), each = (P.s.H + slices - 1) / slices;
  const int pages_each = pages_touched(P.s.rows);
  const int64_t stores = (int64_t)P.s.B * P.s.Hkv * pages_each;
  const int64_t queries = groups * ((P.s.H + each - 1) / each);
  heads_store_kernel<D, DT, PAIRS><<<(unsigned)((stores + 7) / 8 * 8 + (queries + 7) / 8 * 8), 2 * D, 0, stream>>>(
      P, c, slots, cache, scales, pages_each, (int)stores, (int)groups, each);
}

template <int D, int DT>
void store(const HeadsParams& P, const CacheShape& c, const int32_t* slots, uint8_t* cache, float* scales, hipStream_t stream) {
  (P.s.pairs == UGBS_HALVES ? store<D, DT, UGBS_HALVES> : store<D, DT, UGBS_NEIGHBOURS>)(P, c, slots, cache, scales, stream);
}

}  // namespace

hipError_t launch_heads_store(const HeadsParams& P, const CacheShape& c, const int32_t* slots, uint8_t* cache, float* scales,
                              hipStream_t stream) {
  const bool f8 = c.dtype == UGBS_E4M3;
  if (c.d == 64) (f8 ? store<64, UGBS_E4M3> : store<64, UGBS_INT8>)(P, c, slots, cache, scales, stream);
  else if (c.d == 128) (f8 ? store<128, UGBS_E4M3> : store<128, UGBS_INT8>)(P, c, slots, cache, scales, stream);
  else (f8 ? store<256, UGBS_E4M3> : store<256, UGBS_INT8>)(P, c, slots, cache, scales, stream);
  return hipGetLastError();
}

}  // namespace ugbs
