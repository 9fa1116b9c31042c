// Parts of few rows of the attention over the cache: 16 or 32 query rows against pages of a kv head.
//
// A kv head's query rows of a request, r = i G + g (new token i, query head g
// of the G that share the kv head), are taken 16 RT at a time: one tile.  Row r
// sits at position kv_len - q_len + i and sees the keys up to it.  Transposed
// products on 16x16x32 bf16 matrix instructions: S^T = K Q^T, whose result
// leaves 8 keys of one row per lane and 32 keys, and those probabilities,
// packed to bf16, already are the B operand of O^T += V^T P^T.  The cache's
// bytes reach the A operands of both straight from memory (its layout is made
// for it), are widened to bf16 in registers, and their scales go into the
// softmax factor (keys) and the probabilities (values): powers of two, exact.
// Softmax in fp32, base 2, with a running maximum; sums of the probabilities
// before their rounding to bf16 (2^-8 relative at most).
#pragma once
#include <type_traits>

#include "cache_attend.h"

namespace ugbs {
namespace {

// One part: RT tiles of 16 rows (all the rows of a kv head, so a byte is read by
// one wave) against pages p0 .. p1 - 1.  The half pages (32 tokens) go round the
// waves; the waves' sums are joined in LDS at the end.  A wave has one set of
// registers for a half page's bytes: the next keys are asked for when the last
// product with these is issued, the next values likewise, so one of the two is
// always on its way, and the registers leave room for more waves, which hide the
// rest.  Bound by HBM: 32 ragged requests of up to 8K (32/8 heads, d 128, 276 MB)
// 53 us with the join, 5.2 TB/s (large copies reach 4.7 to 6.1); one of 128K (28/4 heads,
// 134 MB) 30.3 us, of which the join 4.6.
//
// Part u against pages p0 .. p1 - 1; its sums go to rows `row` .. of the workspace, or (row < 0) to O.
template <int D, int RT, int NW>
struct RowsMemory {
  __align__(16) float o[NW * 16 * D];
  float2 ml[NW * 16 * RT];
};
template <int D, int DT, int RT, int NW, Mode MODE>
__device__ __forceinline__ void rows_part(const CacheAttendParams& P, const Part& u, int64_t row, int p0, int p1,
                                          RowsMemory<D, RT, NW>& memory) {
  constexpr int L = D / 32;                 // 16-byte loads of a lane: keys, and again values
  constexpr int ROWS = 16 * RT;
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // waves 2 j and 2 j + 1 take the halves of pages p0 + j, p0 + j + NW / 2, ...
  const int half = w & 1;
  Pages pages = pages_of(P, u, p0, p1, w >> 1, NW / 2);

  // this lane's rows: the last key each sees, and its query
  int last[RT];
  bf16x8 bq[RT][2 * (D / 64)];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = u.tile * ROWS + 16 * rt + c16;
    const bool ok = r < u.q * s.G;
    size_t at;
    if constexpr (MODE == kPrefix) {
      const int2 x = row_of(P, u, r);
      last[rt] = x.y;
      at = x.x;
    } else {
      const int i = ok ? r / s.G : 0, h = u.kvh * s.G + (ok ? r % s.G : 0);
      last[rt] = ok ? u.kv - u.q + i : -1;
      at = ((size_t)u.b * s.H + h) * s.rows + i;
    }
    const uint16_t* const q = P.Q + at * D + 16 * g;
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
  int all_see = u.kv - u.q + u.tile * ROWS / s.G;
  if constexpr (MODE == kPrefix) {
    all_see = INT32_MAX;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
      if (u.tile * ROWS + 16 * rt + c16 < u.q * s.G) all_see = min(all_see, last[rt]);
#pragma unroll
    for (int o = 1; o < 16; o *= 2) all_see = min(all_see, __shfl_xor(all_see, o));
    all_see = __builtin_amdgcn_readfirstlane(all_see);
  }

  uint4 kx[L], vx[L];
  auto bytes_of = [&](int page) {
    return reinterpret_cast<const uint4*>(P.cache + ((size_t)page * s.Hkv + u.kvh) * 2 * (kBlock * D) + half * 32 * D) + lane;
  };
  auto fetch_k = [&](int page) {
    const uint4* const src = bytes_of(page);
#pragma unroll
    for (int e = 0; e < L; ++e) kx[e] = load_once(src + 64 * e);
  };
  auto fetch_v = [&](int page) {
    const uint4* const src = bytes_of(page) + kBlock * D / 16;
#pragma unroll
    for (int e = 0; e < L; ++e) vx[e] = load_once(src + 64 * e);
  };

  f32x4 acc[RT][D / 16];
  float m_run[RT], l_run[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[rt] = kNoMax;
    l_run[rt] = 0.f;
  }

  // One half page; MORE: another one follows, whose loads go out here.  (The last one is a
  // step of its own: loads behind a condition would make every wait one for all of them.)
  auto step = [&](int l, int next, auto more_tag) {
    constexpr bool MORE = decltype(more_tag)::value;
    const int key0 = kBlock * pages.at(l) + 32 * half;      // position of the half page's first token
    const float f = pages.key_scale(l) * P.scale_log2, vs = pages.value_scale(l);
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
    if constexpr (MORE) fetch_k(pages.page(next));
    const bool edge = key0 + 31 > all_see;
    bf16x8 bp[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
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
        if (DT != UGBS_E4M3) p[e] *= vs;
      }
      bp[rt] = as_bf16x8(make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])));
    }
    if (key0 + 32 > u.kv) {
      const uint2 keep = live_bytes(u.kv, key0);
#pragma unroll
      for (int e = 0; e < L; ++e) vx[e] = make_uint4(vx[e].x & keep.x, vx[e].y & keep.y, vx[e].z & keep.x, vx[e].w & keep.y);
    }
#pragma unroll
    for (int e = 0; e < L; ++e) {
      const bf16x8 a = operand<DT>(vx[e].x, vx[e].y, vs), b = operand<DT>(vx[e].z, vx[e].w, vs);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc[rt][2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bp[rt], acc[rt][2 * e], 0, 0, 0);
        acc[rt][2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, bp[rt], acc[rt][2 * e + 1], 0, 0, 0);
      }
    }
    if constexpr (MORE) fetch_v(pages.page(next));
  };
  int key_first = INT32_MAX;                // the first position this wave sees
  while (pages.left) {
    int l = pages.pop();
    fetch_k(pages.page(l));
    fetch_v(pages.page(l));
    key_first = min(key_first, kBlock * pages.at(l) + 32 * half);
    while (pages.left) {
      const int next = pages.pop();
      step(l, next, std::true_type{});
      l = next;
    }
    step(l, 0, std::false_type{});
    pages.advance();
  }

  bool seen[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) seen[rt] = key_first <= last[rt];
  finish_part<D, RT, NW>(P, u, row, memory.o, memory.ml, acc, m_run, l_run, seen);
}

}  // namespace
}  // namespace ugbs
