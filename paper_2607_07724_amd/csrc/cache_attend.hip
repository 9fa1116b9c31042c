// Attention of the newest tokens of every request over its cached tokens.
//
// A kv head's query rows of a request, r = i G + g (new token i, query head g
// of the G that share the kv head), are taken 16 at a time: one tile.  Row r
// sits at position kv_len - q_len + i and sees the keys up to it.  Transposed
// products on 16x16x32 bf16 matrix instructions: S^T = K Q^T, whose result
// leaves 8 keys of one row per lane and 32 keys, and those probabilities,
// packed to bf16, already are the B operand of O^T += V^T P^T.  The cache's
// bytes reach the A operands of both straight from memory (its layout is made
// for it), are widened to bf16 in registers, and their scales go into the
// softmax factor (keys) and the probabilities (values): powers of two, exact.
// Softmax in fp32, base 2, with a running maximum; sums of the probabilities
// before their rounding to bf16 (2^-8 relative at most).
//
// Work is split along the pages where there are few rows: with W the pages of
// all tiles, a tile of n pages goes to ceil(n / X) workgroups, X = ceil(W / kTarget)
// (at least kMinPages), so that a long request among short ones does not hold
// up the call.  The lengths are on the device; each wave forms the sums over
// the requests for itself.  Parts leave their sums and maxima in the workspace,
// and a second launch joins them, in the order of the pages.
#include "cache_internal.h"

namespace ugbs {
namespace {

constexpr float kNoMax = -3.402823466e38f;     // a row's maximum before its first key
constexpr int kTarget = 1024;                  // parts a call aims at
constexpr int kMinPages = 8;                   // pages of a part, at least

struct CacheAttendParams {
  CacheShape s;
  const uint16_t* Q;
  const uint8_t* cache;
  const float* scales;
  const int32_t* table;
  const int32_t* kv_lens;
  const int32_t* q_lens;
  uint16_t* O;
  float* part_o;      // [slots][rows of a tile][D]: sums of p v, unnormalised
  float2* part_ml;    // [slots][rows of a tile]: maximum (-inf: no key), sum of p
  float scale_log2;
  bool splits;        // parts are allowed
};

__device__ __forceinline__ int scan_add(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// What a wave knows of a request: rows, tiles, pages.
struct Lengths {
  int q, kv, tiles, pages;
};
template <int ROWS>
__device__ __forceinline__ Lengths lengths_of(const CacheAttendParams& P, int b) {
  Lengths r;
  r.q = min(max(P.q_lens[b], 0), P.s.rows);
  r.kv = min(max(P.kv_lens[b], 0), P.s.max_pages * kBlock);
  r.tiles = (r.q * P.s.G + ROWS - 1) / ROWS;
  r.pages = (r.kv + kBlock - 1) / kBlock;
  return r;
}

struct Part {
  int b, kvh, tile, split, splits, slot, q, kv;   // slot: of the tile's first part
};

// Part number pos of the call (MERGE: tile number pos among the split ones).
// The parts of a request follow each other: kv head, tile, part.  Uniform over the wave.
template <int ROWS, bool MERGE>
__device__ bool find_part(const CacheAttendParams& P, int pos, Part* out) {
  const int lane = threadIdx.x & 63, B = P.s.B, Hkv = P.s.Hkv;
  int per = kMinPages;
  if (P.splits) {
    // tiles * pages <= 2^30 in sum over a wave's lane? held in 64 bits
    unsigned long long w = 0;
    for (int b = lane; b < B; b += 64) {
      const Lengths r = lengths_of<ROWS>(P, b);
      w += (unsigned long long)r.tiles * r.pages;
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const unsigned lo = __shfl_xor((unsigned)w, o), hi = __shfl_xor((unsigned)(w >> 32), o);
      w += (unsigned long long)hi << 32 | lo;
    }
    w = (w * Hkv + kTarget - 1) / kTarget;
    per = w > UGBS_MAX_BLOCKS ? UGBS_MAX_BLOCKS : w > kMinPages ? (int)w : kMinPages;
  }
  int before = 0, slots = 0;
  for (int c = 0; c < B; c += 64) {
    Lengths r{0, 0, 0, 0};
    int splits = 1;
    if (c + lane < B) {
      r = lengths_of<ROWS>(P, c + lane);
      if (P.splits && r.pages > per) splits = (r.pages + per - 1) / per;
    }
    const int units = r.tiles * Hkv;
    const int used = splits > 1 ? units * splits : 0;
    const int mine = MERGE ? (splits > 1 ? units : 0) : units * splits;
    const int upto = before + scan_add(mine), slots_upto = slots + scan_add(used);
    const unsigned long long found = __ballot(pos >= upto - mine && pos < upto);
    if (found) {
      const int l = __builtin_ctzll(found);
      out->b = c + l;
      out->q = __shfl(r.q, l);
      out->kv = __shfl(r.kv, l);
      out->splits = __shfl(splits, l);
      const int tiles = __shfl(r.tiles, l);
      int at = pos - __shfl(upto - mine, l);
      out->split = 0;
      if (!MERGE) {
        out->split = at % out->splits;
        at /= out->splits;
      }
      out->slot = __shfl(slots_upto - used, l) + at * out->splits;
      out->tile = at % tiles;
      out->kvh = at / tiles;
      return true;
    }
    before = __shfl(upto, 63);
    slots = __shfl(slots_upto, 63);
  }
  return false;
}

// Pages that rows tile 16 .. + 15 see (the last row sees most).
template <int ROWS>
__device__ __forceinline__ int pages_seen(const CacheAttendParams& P, const Part& u) {
  const int last = min((u.tile + 1) * ROWS, u.q * P.s.G) - 1;
  const int end = u.kv - u.q + last / P.s.G + 1;          // keys the last row sees
  return end <= 0 ? 0 : (end + kBlock - 1) / kBlock;
}

__device__ __forceinline__ float sum_groups(float x) {    // over the four lanes that hold a row
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// One part: 16 rows against pages p0 .. p1 - 1.  The half pages (32 tokens) go
// round the waves, each of which has the next one's bytes in flight while it
// computes; the waves' sums are joined in LDS at the end.
template <int D, int DT, int NW>
__global__ void __launch_bounds__(64 * NW) cache_attend_rows_kernel(CacheAttendParams P) {
  constexpr int L = D / 32;                 // 16-byte loads of a lane: keys, and again values
  constexpr int ROWS = 16;
  __shared__ __align__(16) float s_o[NW][ROWS][D + 4];
  __shared__ float2 s_ml[NW][ROWS];
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Part u;
  if (!find_part<ROWS, false>(P, blockIdx.x, &u)) return;
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.kvh = __builtin_amdgcn_readfirstlane(u.kvh);
  const int n = pages_seen<ROWS>(P, u);
  const int p0 = (int)((long long)n * u.split / u.splits), p1 = (int)((long long)n * (u.split + 1) / u.splits);

  // this lane's row: new token i, query head h; the last key it sees
  const int r = u.tile * ROWS + c16;
  const bool row_ok = r < u.q * s.G;
  const int i = row_ok ? r / s.G : 0, h = u.kvh * s.G + (row_ok ? r % s.G : 0);
  const int last = row_ok ? u.kv - u.q + i : -1;
  // every valid row sees the keys up to here
  const int all_see = u.kv - u.q + u.tile * ROWS / s.G;
  const size_t qo = (((size_t)u.b * s.H + h) * s.rows + i) * D;
  bf16x8 bq[2 * (D / 64)];
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row_ok) v = *reinterpret_cast<const uint4*>(P.Q + qo + 64 * x + 16 * g + 8 * y);
      bq[2 * x + y] = as_bf16x8(v);
    }

  const int32_t* const row = P.table + (size_t)u.b * s.max_pages;
  struct Half {
    uint4 k[L], v[L];
    float ks, vs;
    bool there;
  };
  auto fetch = [&](int at, Half& x) {       // half page `at` of the request
    const int page = __builtin_amdgcn_readfirstlane(row[at >> 1]);
    x.there = page >= 0 && page < s.n_pages;
    if (!x.there) return;
    const size_t ph = (size_t)page * s.Hkv + u.kvh;
    const uint4* const src = reinterpret_cast<const uint4*>(P.cache + ph * 2 * (kBlock * D) + (at & 1) * 32 * D) + lane;
#pragma unroll
    for (int e = 0; e < L; ++e) x.k[e] = src[64 * e];
#pragma unroll
    for (int e = 0; e < L; ++e) x.v[e] = src[kBlock * D / 16 + 64 * e];
    x.ks = P.scales[2 * ph];
    x.vs = P.scales[2 * ph + 1];
  };

  f32x4 acc[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;
  bool seen = false;                        // a key of this row has been looked at

  auto step = [&](int at, Half& x) {
    if (!x.there) return;
    const int key0 = 32 * at;               // position of the half page's first token
    f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const uint4 raw = x.k[kt * (D / 64) + e];
        sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand<DT>(raw.x, raw.y), bq[2 * e], sc[kt], 0, 0, 0);
        sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand<DT>(raw.z, raw.w), bq[2 * e + 1], sc[kt], 0, 0, 0);
      }
    const float f = x.ks * P.scale_log2;
    const bool edge = key0 + 31 > all_see;
    seen |= key0 <= last;
    float mx = kNoMax;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y = sc[kt][e] * f;
        if (edge && key0 + 16 * kt + 4 * g + e > last) y = -__builtin_huge_valf();
        sc[kt][e] = y;
        mx = fmaxf(mx, y);
      }
    const float m_new = fmaxf(m_run, rows_max(mx));
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[dt][e] *= alpha;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(sc[e >> 2][e & 3] - m_run);
      l_run += p[e];
      p[e] *= x.vs;
    }
    const bf16x8 bp = as_bf16x8(make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])));
    // bytes behind the last token may be anything: 0 (a probability of 0 does not make them harmless)
    uint32_t keep[2] = {~0u, ~0u};
    if (key0 + 32 > u.kv) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int left = u.kv - (key0 + 16 * kt + 4 * g);
        keep[kt] = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
      }
    }
#pragma unroll
    for (int e = 0; e < L; ++e) {
      acc[2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand<DT>(x.v[e].x & keep[0], x.v[e].y & keep[1]), bp, acc[2 * e], 0, 0, 0);
      acc[2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand<DT>(x.v[e].z & keep[0], x.v[e].w & keep[1]), bp, acc[2 * e + 1], 0, 0, 0);
    }
  };

  const int end = 2 * p1;
  int at = 2 * p0 + w;
  Half x, y;
  if (at < end) fetch(at, x);
  for (; at < end; at += 2 * NW) {
    const bool more = at + NW < end;
    if (more) fetch(at + NW, y);
    step(at, x);
    if (!more) break;
    if (at + 2 * NW < end) fetch(at + 2 * NW, x);
    step(at + NW, y);
  }

  // ---- the waves' sums
  const float l_row = sum_groups(l_run);
  if (g == 0) s_ml[w][c16] = make_float2(seen ? m_run : -__builtin_huge_valf(), l_row);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(&s_o[w][c16][16 * dt + 4 * g]) = acc[dt];
  __syncthreads();
  constexpr int CG = D / 4;                 // 4 channels a thread
  for (int k = tid; k < ROWS * CG; k += 64 * NW) {
    const int rr = k / CG, c = 4 * (k % CG);
    const int at_row = u.tile * ROWS + rr;
    if (at_row >= u.q * s.G) continue;
    float M = -__builtin_huge_valf();
#pragma unroll
    for (int v = 0; v < NW; ++v) M = fmaxf(M, s_ml[v][rr].x);
    float l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float2 ml = s_ml[v][rr];
      if (ml.x == -__builtin_huge_valf()) continue;       // this wave saw none of the row's keys
      const float a = __builtin_amdgcn_exp2f(ml.x - M);
      l += a * ml.y;
      const f32x4 ov = *reinterpret_cast<const f32x4*>(&s_o[v][rr][c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += a * ov[e];
    }
    if (u.splits == 1) {
      const int ii = at_row / s.G, hh = u.kvh * s.G + at_row % s.G;
      // no key: 0; (every score -inf: NaN, as its softmax is)
      const float inv = M == -__builtin_huge_valf() ? 0.f : l != 0.f ? 1.0f / l : __builtin_nanf("");
      *reinterpret_cast<uint2*>(P.O + (((size_t)u.b * s.H + hh) * s.rows + ii) * D + c) =
          make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    } else {
      const size_t slot = (size_t)u.slot + u.split;
      *reinterpret_cast<f32x4*>(P.part_o + (slot * ROWS + rr) * D + c) = o;
      if (c == 0) P.part_ml[slot * ROWS + rr] = make_float2(M, l);
    }
  }
}

// Joins the parts of one row: one workgroup of D / 4 threads per (split tile, row).
template <int D, int ROWS>
__global__ void __launch_bounds__(64) cache_join_kernel(CacheAttendParams P) {
  Part u;
  if (!find_part<ROWS, true>(P, blockIdx.x, &u)) return;
  const CacheShape& s = P.s;
  const int rr = blockIdx.y, at_row = u.tile * ROWS + rr, c = 4 * threadIdx.x;
  if (at_row >= u.q * s.G || c >= D) return;
  const float2* const ml = P.part_ml + (size_t)u.slot * ROWS + rr;
  float M = -__builtin_huge_valf();
  for (int v = 0; v < u.splits; ++v) M = fmaxf(M, ml[v * ROWS].x);
  float l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int v = 0; v < u.splits; ++v) {
    const float2 x = ml[v * ROWS];
    if (x.x == -__builtin_huge_valf()) continue;
    const float a = __builtin_amdgcn_exp2f(x.x - M);
    l += a * x.y;
    const f32x4 ov = *reinterpret_cast<const f32x4*>(P.part_o + (((size_t)u.slot + v) * ROWS + rr) * D + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += a * ov[e];
  }
  const float inv = M == -__builtin_huge_valf() ? 0.f : l != 0.f ? 1.0f / l : __builtin_nanf("");
  const int i = at_row / s.G, h = u.kvh * s.G + at_row % s.G;
  *reinterpret_cast<uint2*>(P.O + (((size_t)u.b * s.H + h) * s.rows + i) * D + c) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

int64_t tiles_bound(const CacheShape& s, int rows_of_a_tile) {
  return (int64_t)s.B * s.Hkv * (((int64_t)s.rows * s.G + rows_of_a_tile - 1) / rows_of_a_tile);
}

// Every split tile has at least two parts, and parts of split tiles are at most twice W / X <= kTarget.
constexpr int kSlots = 2 * kTarget;

bool may_split(const CacheShape& s) { return s.max_pages > kMinPages; }

template <int D, int DT>
hipError_t attend_rows(const CacheAttendParams& P, hipStream_t stream) {
  constexpr int NW = 4;
  const int64_t units = tiles_bound(P.s, 16);
  cache_attend_rows_kernel<D, DT, NW><<<(unsigned)(units + (P.splits ? kTarget : 0)), 64 * NW, 0, stream>>>(P);
  if (P.splits) {
    const dim3 grid((unsigned)(units < kTarget ? units : kTarget), 16);
    cache_join_kernel<D, 16><<<grid, 64, 0, stream>>>(P);
  }
  return hipGetLastError();
}

}  // namespace

size_t cache_attend_workspace(const CacheShape& s) {
  return may_split(s) ? (size_t)kSlots * 16 * (s.d * sizeof(float) + sizeof(float2)) : 0;
}

hipError_t launch_cache_attend(const CacheShape& s, const uint16_t* Q, const uint8_t* cache, const float* scales,
                               const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens, uint16_t* O,
                               void* workspace, hipStream_t stream) {
  CacheAttendParams P{s, Q, cache, scales, table, kv_lens, q_lens, O, nullptr, nullptr, 0.f, false};
  P.scale_log2 = s.scale * 1.4426950408889634f;
  P.splits = may_split(s);
  P.part_o = static_cast<float*>(workspace);
  P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)kSlots * 16 * s.d);
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) return f8 ? attend_rows<64, UGBS_E4M3>(P, stream) : attend_rows<64, UGBS_INT8>(P, stream);
  if (s.d == 128) return f8 ? attend_rows<128, UGBS_E4M3>(P, stream) : attend_rows<128, UGBS_INT8>(P, stream);
  return f8 ? attend_rows<256, UGBS_E4M3>(P, stream) : attend_rows<256, UGBS_INT8>(P, stream);
}

}  // namespace ugbs
