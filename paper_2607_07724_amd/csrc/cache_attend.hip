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
constexpr int kTarget = 512;                   // parts a call aims at
constexpr int kMinPages = 8;                   // pages of a part, at least
// Every split tile has at least two parts, and parts of split tiles are at most twice W / X <= kTarget.
constexpr int kSlots = 2 * kTarget;

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

// 1 / l, for a row with maximum M: 0 where it saw no key, NaN where every score was -inf (as its softmax is).
__device__ __forceinline__ float reciprocal(float M, float l) {
  return M == -__builtin_huge_valf() ? 0.f : l != 0.f ? 1.0f / l : __builtin_nanf("");
}

__device__ __forceinline__ float sum_groups(float x) {    // over the four lanes that hold a row
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// One part: RT tiles of 16 rows against pages p0 .. p1 - 1.  The half pages (32
// tokens) go round the waves; the waves' sums are joined in LDS at the end.  A
// wave has one set of registers for a half page's bytes: the next keys are asked
// for when the last product with these is issued, the next values likewise, so
// one of the two is always on its way, and the registers leave room for more
// waves, which hide the rest.
template <int D, int DT, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) cache_attend_rows_kernel(CacheAttendParams P) {
  constexpr int L = D / 32;                 // 16-byte loads of a lane: keys, and again values
  constexpr int ROWS = 16 * RT;
  __shared__ __align__(16) float s_o[NW][16][D + 4];
  __shared__ float2 s_ml[NW][ROWS];
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Part u;
  if (!find_part<ROWS, false>(P, blockIdx.x, &u)) return;
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.kvh = __builtin_amdgcn_readfirstlane(u.kvh);
  u.kv = __builtin_amdgcn_readfirstlane(u.kv);
  const int n = pages_seen<ROWS>(P, u);
  const int p0 = __builtin_amdgcn_readfirstlane((int)((long long)n * u.split / u.splits));
  const int p1 = __builtin_amdgcn_readfirstlane((int)((long long)n * (u.split + 1) / u.splits));

  // this lane's rows: the last key each sees, and its query
  int last[RT];
  bf16x8 bq[RT][2 * (D / 64)];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = u.tile * ROWS + 16 * rt + c16;
    const bool ok = r < u.q * s.G;
    const int i = ok ? r / s.G : 0, h = u.kvh * s.G + (ok ? r % s.G : 0);
    last[rt] = ok ? u.kv - u.q + i : -1;
    const uint16_t* const q = P.Q + (((size_t)u.b * s.H + h) * s.rows + i) * D + 16 * g;
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (ok) v = *reinterpret_cast<const uint4*>(q + 64 * x + 8 * y);
        bq[rt][2 * x + y] = as_bf16x8(v);
      }
  }
  // every valid row sees the keys up to here
  const int all_see = u.kv - u.q + u.tile * ROWS / s.G;

  const int32_t* const row = P.table + (size_t)u.b * s.max_pages;
  uint4 kx[L], vx[L];
  float ks = 0.f, vs = 0.f;                 // scales of the bytes in kx and vx
  auto there = [&](int page) { return page >= 0 && page < s.n_pages; };
  auto half_of = [&](int page, int at) {
    return reinterpret_cast<const uint4*>(P.cache + ((size_t)page * s.Hkv + u.kvh) * 2 * (kBlock * D) + (at & 1) * 32 * D) + lane;
  };
  auto fetch_k = [&](int page, int at) {
    const uint4* const src = half_of(page, at);
#pragma unroll
    for (int e = 0; e < L; ++e) kx[e] = src[64 * e];
  };
  auto fetch_v = [&](int page, int at) {
    const uint4* const src = half_of(page, at) + kBlock * D / 16;
#pragma unroll
    for (int e = 0; e < L; ++e) vx[e] = src[64 * e];
  };

  f32x4 acc[RT][D / 16];
  float m_run[RT], l_run[RT];
  bool seen[RT];                            // a key of the row has been looked at
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[rt] = kNoMax;
    l_run[rt] = 0.f;
    seen[rt] = false;
  }

  // half pages at, at + NW, ... of the request; those in no page are passed over
  const int end = 2 * p1;
  auto next_half = [&](int at, int* page) {
    for (; at < end; at += NW) {
      *page = __builtin_amdgcn_readfirstlane(row[at >> 1]);
      if (there(*page)) break;
    }
    return at;
  };
  int page = 0, page2 = 0;
  int at = next_half(2 * p0 + w, &page);
  if (at < end) {
    fetch_k(page, at);
    fetch_v(page, at);
  }
  while (at < end) {
    const int key0 = 32 * at;               // position of the half page's first token
    const float* const sc_page = P.scales + 2 * ((size_t)page * s.Hkv + u.kvh);
    ks = sc_page[0];
    vs = sc_page[1];
    const int at2 = next_half(at + NW, &page2);
    f32x4 sc[RT][2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) sc[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const uint4 raw = kx[kt * (D / 64) + e];
        const bf16x8 a = operand<DT>(raw.x, raw.y), b = operand<DT>(raw.z, raw.w);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bq[rt][2 * e], sc[rt][kt], 0, 0, 0);
          sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, bq[rt][2 * e + 1], sc[rt][kt], 0, 0, 0);
        }
      }
    }
    if (at2 < end) fetch_k(page2, at2);
    const float f = ks * P.scale_log2;
    const bool edge = key0 + 31 > all_see;
    bf16x8 bp[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      seen[rt] |= key0 <= last[rt];
      float mx = kNoMax;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = sc[rt][kt][e] * f;
          if (edge && key0 + 16 * kt + 4 * g + e > last[rt]) y = -__builtin_huge_valf();
          sc[rt][kt][e] = y;
          mx = fmaxf(mx, y);
        }
      // the maximum moves when a row's exceeds it (asked per lane first)
      if (__ballot(mx > m_run[rt])) {
        const float m_new = fmaxf(m_run[rt], rows_max(mx));
        const float alpha = __builtin_amdgcn_exp2f(m_run[rt] - m_new);
        m_run[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[rt][dt][e] *= alpha;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(sc[rt][e >> 2][e & 3] - m_run[rt]);
        l_run[rt] += p[e];
        p[e] *= vs;
      }
      bp[rt] = as_bf16x8(make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])));
    }
    // bytes behind the last token may be anything: 0 (a probability of 0 does not make them harmless)
    if (key0 + 32 > u.kv) {
      uint32_t keep[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int left = u.kv - (key0 + 16 * kt + 4 * g);
        keep[kt] = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
      }
#pragma unroll
      for (int e = 0; e < L; ++e) vx[e] = make_uint4(vx[e].x & keep[0], vx[e].y & keep[1], vx[e].z & keep[0], vx[e].w & keep[1]);
    }
#pragma unroll
    for (int e = 0; e < L; ++e) {
      const bf16x8 a = operand<DT>(vx[e].x, vx[e].y), b = operand<DT>(vx[e].z, vx[e].w);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc[rt][2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bp[rt], acc[rt][2 * e], 0, 0, 0);
        acc[rt][2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, bp[rt], acc[rt][2 * e + 1], 0, 0, 0);
      }
    }
    if (at2 < end) fetch_v(page2, at2);
    at = at2;
    page = page2;
  }

  // ---- the waves' sums, 16 rows at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = sum_groups(l_run[rt]);
    if (g == 0) s_ml[w][16 * rt + c16] = make_float2(seen[rt] ? m_run[rt] : -__builtin_huge_valf(), l);
  }
  constexpr int CG = D / 4;                 // 4 channels a thread
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(&s_o[w][c16][16 * dt + 4 * g]) = acc[rt][dt];
    __syncthreads();
    for (int k = tid; k < 16 * CG; k += 64 * NW) {
      const int r16 = k / CG, c = 4 * (k % CG), rr = 16 * rt + r16;
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
        if (ml.x == -__builtin_huge_valf()) continue;     // this wave saw none of the row's keys
        const float a = __builtin_amdgcn_exp2f(ml.x - M);
        l += a * ml.y;
        const f32x4 ov = *reinterpret_cast<const f32x4*>(&s_o[v][r16][c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += a * ov[e];
      }
      if (u.splits == 1) {
        const int i = at_row / s.G, h = u.kvh * s.G + at_row % s.G;
        const float inv = reciprocal(M, l);
        *reinterpret_cast<uint2*>(P.O + (((size_t)u.b * s.H + h) * s.rows + i) * D + c) =
            make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
      } else {
        const size_t slot = (size_t)u.slot + u.split;
        *reinterpret_cast<f32x4*>(P.part_o + (slot * ROWS + rr) * D + c) = o;
        if (c == 0) P.part_ml[slot * ROWS + rr] = make_float2(M, l);
      }
    }
  }
}

// Joins the parts of one row: a workgroup per (split tile, row), D / 4 threads to
// a part, the parts round the others.
constexpr int kJoin = 256;
template <int D, int ROWS>
__global__ void __launch_bounds__(kJoin) cache_join_kernel(CacheAttendParams P) {
  constexpr int CG = D / 4, GR = kJoin / CG;
  __shared__ float s_w[kSlots];             // weights of the parts
  __shared__ float2 s_ml[kJoin / 64];
  __shared__ f32x4 s_o[GR][CG];
  Part u;
  if (!find_part<ROWS, true>(P, blockIdx.x, &u)) return;
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, w = tid >> 6, rr = blockIdx.y, at_row = u.tile * ROWS + rr;
  if (at_row >= u.q * s.G) return;
  const float2* const ml = P.part_ml + (size_t)u.slot * ROWS + rr;
  float M = -__builtin_huge_valf();
  for (int v = tid; v < u.splits; v += kJoin) {
    const float m = ml[(size_t)v * ROWS].x;
    s_w[v] = m;
    M = fmaxf(M, m);
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) s_ml[w].x = M;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kJoin / 64; ++v) M = fmaxf(M, s_ml[v].x);
  float l = 0.f;
  for (int v = tid; v < u.splits; v += kJoin) {
    const float a = s_w[v] == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(s_w[v] - M);
    s_w[v] = a;
    if (a != 0.f) l += a * ml[(size_t)v * ROWS].y;
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) l += __shfl_xor(l, o);
  if ((tid & 63) == 0) s_ml[w].y = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int v = 0; v < kJoin / 64; ++v) l += s_ml[v].y;
  const int gr = tid / CG, c = tid % CG;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4* const po = reinterpret_cast<const f32x4*>(P.part_o + ((size_t)u.slot * ROWS + rr) * D) + c;
#pragma unroll 4
  for (int v = gr; v < u.splits; v += GR) {
    const float a = s_w[v];
    const f32x4 x = po[(size_t)v * (ROWS * CG)];
    // (a part that saw none of the row's keys has written zeros)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += a * x[e];
  }
  s_o[gr][c] = o;
  __syncthreads();
  if (gr == 0) {
#pragma unroll
    for (int v = 1; v < GR; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += s_o[v][c][e];
    const float inv = reciprocal(M, l);
    const int i = at_row / s.G, h = u.kvh * s.G + at_row % s.G;
    *reinterpret_cast<uint2*>(P.O + (((size_t)u.b * s.H + h) * s.rows + i) * D + 4 * c) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
  }
}

int64_t tiles_bound(const CacheShape& s, int rows_of_a_tile) {
  return (int64_t)s.B * s.Hkv * (((int64_t)s.rows * s.G + rows_of_a_tile - 1) / rows_of_a_tile);
}

bool may_split(const CacheShape& s) { return s.max_pages > kMinPages; }

template <int D, int DT, int RT>
hipError_t attend_rows(const CacheAttendParams& P, hipStream_t stream) {
  constexpr int NW = 4, ROWS = 16 * RT;
  const int64_t units = tiles_bound(P.s, ROWS);
  cache_attend_rows_kernel<D, DT, RT, NW><<<(unsigned)(units + (P.splits ? kTarget : 0)), 64 * NW, 0, stream>>>(P);
  if (P.splits) {
    const int64_t rows = (int64_t)P.s.rows * P.s.G;
    const dim3 grid((unsigned)(units < kTarget ? units : kTarget), (unsigned)(rows < ROWS ? rows : ROWS));
    cache_join_kernel<D, ROWS><<<grid, kJoin, 0, stream>>>(P);
  }
  return hipGetLastError();
}

// Rows of a tile: as many as the call can have, up to 32.
int tile_rows(const CacheShape& s) { return (int64_t)s.rows * s.G <= 16 ? 16 : 32; }

template <int D, int DT>
hipError_t attend(const CacheAttendParams& P, hipStream_t stream) {
  return tile_rows(P.s) == 16 ? attend_rows<D, DT, 1>(P, stream) : attend_rows<D, DT, 2>(P, stream);
}

}  // namespace

size_t cache_attend_workspace(const CacheShape& s) {
  return may_split(s) ? (size_t)kSlots * tile_rows(s) * (s.d * sizeof(float) + sizeof(float2)) : 0;
}

hipError_t launch_cache_attend(const CacheShape& s, const uint16_t* Q, const uint8_t* cache, const float* scales,
                               const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens, uint16_t* O,
                               void* workspace, hipStream_t stream) {
  CacheAttendParams P{s, Q, cache, scales, table, kv_lens, q_lens, O, nullptr, nullptr, 0.f, false};
  P.scale_log2 = s.scale * 1.4426950408889634f;
  P.splits = may_split(s);
  P.part_o = static_cast<float*>(workspace);
  P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)kSlots * tile_rows(s) * s.d);
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) return f8 ? attend<64, UGBS_E4M3>(P, stream) : attend<64, UGBS_INT8>(P, stream);
  if (s.d == 128) return f8 ? attend<128, UGBS_E4M3>(P, stream) : attend<128, UGBS_INT8>(P, stream);
  return f8 ? attend<256, UGBS_E4M3>(P, stream) : attend<256, UGBS_INT8>(P, stream);
}

}  // namespace ugbs
