// From a projection's rows to heads: the norm of a query or key head, its rotation by
// position, and the launchers of the kernels.
//
// A row is the d channels of one head of one token.  d / 16 lanes hold it, 16 channels
// each, as two eights, 8 l .. 8 l + 7 and as many half the rotated channels further on; the other
// channels' likewise.  So the lanes' first eights follow each other, as do their second ones (a
// store of every other 16 bytes costs: 15000 tokens of 16/2 heads, d 256, 66 us for 57; runs that are no
// whole lines, as those of rot 64, still 2 of these), and a lane rotates by itself, whichever way channels
// are paired, with 8 angles.
//   y = x / sqrt(mean x^2 + eps) * w,   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
// in fp32, rounded to bf16 once at the end.  Products and sums are written as the
// operations they are (no contraction left to the compiler), so that every kernel that
// takes a row gives the same bits.
#pragma once
#include "cache_internal.h"

namespace ugbs {

struct HeadsShape {
  int B, H, Hkv, d, rows, rot, pairs, axes;
  float eps, gain;
};

struct HeadsParams {
  HeadsShape s;
  ugbs_rows q, k, v;
  const float* q_norm;
  const float* k_norm;
  const double* freqs;
  const int32_t* axis;
  const int32_t* positions;
  const int32_t* first;
  const int32_t* lens;
  uint16_t* Q;
  uint16_t* K;
  uint16_t* V;
};

hipError_t launch_heads_split(const HeadsParams& P, hipStream_t stream);
hipError_t launch_heads_store(const HeadsParams& P, const CacheShape& c, const int32_t* slots, uint8_t* cache, float* scales,
                              hipStream_t stream);

namespace {

// An angle in turns, modulo one, in units of 2^-64: what a position adds to it (whole turns that a frequency has per
// position are whole turns at every position).  Of a negative one the turns are those of its opposite, backwards: the
// fraction itself would lie just below one, where 53 bits leave 2^-54 of a turn at each position.
__device__ __forceinline__ uint64_t turns_of(double f) {
  const uint64_t t = (uint64_t)(__builtin_amdgcn_fract(fabs(f) * 0.15915494309189535) * 18446744073709551616.0);      // (fract is below one)
  return f < 0.0 ? 0 - t : t;
}

// (cos, sin) of an angle, times gain: the nearest quarter turn, and what is left, 2 pi y with |y| <= 1/8, by the
// Taylor series, which end 1e-10 (cos) and 2e-9 (sin) off at an eighth.
__device__ __forceinline__ float2 turned(uint64_t turns, float gain) {
  const uint32_t u = (uint32_t)(turns >> 32), n = (u + (1u << 29)) >> 30;
  const float x = (float)(int)(u - (n << 30)) * 1.4629180792671596e-9f;                // 2 pi / 2^32
  const float z = x * x;
  float s = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = __builtin_fmaf(z, s, 8.3333333e-3f);
  s = __builtin_fmaf(z, s, -1.6666667e-1f);
  s = __builtin_fmaf(z * x, s, x);
  float c = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = __builtin_fmaf(z, c, -1.3888889e-3f);
  c = __builtin_fmaf(z, c, 4.1666667e-2f);
  c = __builtin_fmaf(z, c, -0.5f);
  c = __builtin_fmaf(z, c, 1.0f);
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_float2((n + 1 & 2 ? -a : a) * gain, (n & 2 ? -b : b) * gain);
}

// Angles of tokens into LDS, [token][rot / 2], by THREADS threads, each of which takes one pair of channels.
template <int THREADS>
struct Angles {
  int half, j, t0, at_once, axis;
  double f;
  // (its loads are asked for early, and waited for when angles are formed)
  __device__ __forceinline__ explicit Angles(const HeadsParams& P) {
    half = P.s.rot / 2;
    j = t0 = at_once = axis = 0;
    f = 0.0;
    if (half == 0) return;
    j = (int)threadIdx.x % half;
    t0 = (int)threadIdx.x / half;
    at_once = THREADS / half;
    f = P.freqs[j];
    if (P.positions && P.axis) axis = min(max(P.axis[j], 0), P.s.axes - 1);
  }
  // Tokens from .. behind - 1.  token(t): its request and row.
  template <class Token>
  __device__ __forceinline__ void fill(const HeadsParams& P, int from, int behind, Token token, float2* s_angle) const {
    if (t0 >= at_once) return;
    const uint64_t step = turns_of(f);
    for (int t = from + t0; t < behind; t += at_once) {
      const int2 x = token(t);
      int64_t pos;
      if (P.positions) pos = P.positions[((size_t)axis * P.s.B + x.x) * P.s.rows + x.y];
      else pos = (int64_t)(P.first ? P.first[x.x] : 0) + x.y;
      s_angle[t * half + j] = turned((uint64_t)pos * step, P.s.gain);
    }
  }
};

__device__ __forceinline__ int rows_of(const HeadsParams& P, int b) {
  return P.lens ? min(max(P.lens[b], 0), P.s.rows) : P.s.rows;
}

// Where the eights of lane l of a row lie.
__device__ __forceinline__ int2 eights_of(const HeadsShape& s, int l) {
  const bool rotated = 16 * l < s.rot;
  const int first = rotated ? 0 : s.rot, n = rotated ? s.rot : s.d - s.rot, at = first + 8 * (l - first / 16);    // among these n channels
  return make_int2(at, at + n / 2);
}

// The angles of lane l, which lie in a row of rot / 2: pairs of channels c and c + rot / 2, or 2 j and 2 j + 1.
template <int PAIRS>
__device__ __forceinline__ void angles_of(const HeadsShape& s, const float2* row, int l, float2 (&cs)[8]) {
  if (16 * l >= s.rot) l = 0;
  const int second = PAIRS == UGBS_HALVES ? 8 * l + 4 : s.rot / 4 + 4 * l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 y = reinterpret_cast<const float4*>(row + (e < 2 ? (PAIRS == UGBS_HALVES ? 8 * l : 4 * l) : second))[e & 1];
    cs[2 * e] = make_float2(y.x, y.y);
    cs[2 * e + 1] = make_float2(y.z, y.w);
  }
}

// 16 bytes that the next kernel reads, if they are still there: nothing here does.
__device__ __forceinline__ void store_through(uint16_t* to, uint4 v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(to));
}

// Workgroup j of n runs on XCD j mod 8: its place such that each XCD has a share in a row.
__device__ __forceinline__ int place_in_row(int j, int n) {
  const int x = j % 8, q = n / 8, r = n % 8;
  return x * q + min(x, r) + j / 8;
}

// Sum over the LANES lanes of a row (4, 8 or 16, all active).
template <int LANES>
__device__ __forceinline__ float sum_row(float x) {
  auto add = [&](int y) { x += __uint_as_float((unsigned)y); };
  add(dpp<0xb1, 0xf>((int)__float_as_uint(x)));                       // lane ^ 1
  add(dpp<0x4e, 0xf>((int)__float_as_uint(x)));                       // lane ^ 2
  if (LANES >= 8) add(dpp<0x141, 0xf>((int)__float_as_uint(x)));      // 7 - lane, within 8
  if (LANES >= 16) add(dpp<0x140, 0xf>((int)__float_as_uint(x)));     // 15 - lane, within 16
  return x;
}

__device__ __forceinline__ void unpack8(uint4 v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// One row: this lane's eights a, b.  w: their 16 weights (NORM).  All lanes of the row are active.
template <int D, int PAIRS, bool NORM>
__device__ __forceinline__ void do_row(uint4& a, uint4& b, const float (&w)[16], const float2 (&cs)[8], bool rotated, float eps) {
  float x[16];
  unpack8(a, x);
  unpack8(b, x + 8);
  if constexpr (NORM) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
    sum = sum_row<D / 16>(sum);
    const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / D, eps));
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = x[e] * r * w[e];
  }
  if (rotated) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      constexpr bool H = PAIRS == UGBS_HALVES;
      const int p = H ? j : 2 * j, q = H ? j + 8 : 2 * j + 1;
      const float u = x[p], v = x[q];
      x[p] = __builtin_fmaf(u, cs[j].x, -(v * cs[j].y));
      x[q] = __builtin_fmaf(v, cs[j].x, u * cs[j].y);
    }
  }
  a = pack8(x);
  b = pack8(x + 8);
}

__device__ __forceinline__ void weights_of(const float* norm, int2 c, float (&w)[16]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 y = *reinterpret_cast<const float4*>(norm + (e < 2 ? c.x : c.y) + 4 * (e & 1));
    w[4 * e] = y.x;
    w[4 * e + 1] = y.y;
    w[4 * e + 2] = y.z;
    w[4 * e + 3] = y.w;
  }
}

__device__ __forceinline__ const uint16_t* row_at(const ugbs_rows& r, int b, int i, int h) {
  return static_cast<const uint16_t*>(r.at) + b * r.batch + i * r.token + h * r.head;
}

// Tokens of a wave: 1024 / d rows of one head at a time.
template <int D>
constexpr int kTokens = 1024 / D;

// Heads h0 .. h1 - 1 of the queries, keys and values, in this order, of tokens n0 .. of the batch:
// the work of a workgroup of NW waves.  A wave takes a head of kTokens tokens at a time, whose
// rows follow each other in the result (1 to 2 KiB in a row).  The angles are formed once, in LDS,
// and stay in registers over the heads.
template <int D, int PAIRS, int NW>
__device__ __forceinline__ void split_heads(const HeadsParams& P, int n0, int h0, int h1, float2* s_angle) {
  constexpr int LANES = D / 16, T = kTokens<D>;
  const HeadsShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane % LANES, total = s.B * s.rows, half = s.rot / 2;
  const int t = lane / LANES, n = min(n0 + t, total - 1), b = n / s.rows, i = n % s.rows;
  const bool live = n0 + t < total && i < rows_of(P, b), rotated = 16 * l < s.rot;
  float2 cs[8];
  if (s.rot > 0 && h0 < s.H + s.Hkv) {
    Angles<64 * NW>(P).fill(P, 0, T, [&](int x) {
      const int at = min(n0 + x, total - 1);
      return make_int2(at / s.rows, at % s.rows);
    }, s_angle);
    __syncthreads();
    angles_of<PAIRS>(s, s_angle + t * half, l, cs);
  }
  const int2 c = eights_of(s, l);
  int h = h0 + w;
  auto part = [&](const ugbs_rows& from, uint16_t* to, const float* norm, int before, int heads, bool turn) {
    if (h >= min(h1, before + heads)) return;
    float wt[16];
    if (norm) weights_of(norm, c, wt);
    const uint16_t* const x = row_at(from, b, i, 0);
    uint16_t* const y = to + ((size_t)b * heads * s.rows + i) * D;
    // the next head's row is on its way while this one is worked on
    const int end = min(h1, before + heads);
    uint4 u, v, u2 = make_uint4(0, 0, 0, 0), v2 = u2;
    auto fetch = [&](int at_head, uint4& a, uint4& b) {
      const uint16_t* const at = x + (int64_t)(at_head - before) * from.head;
      a = *reinterpret_cast<const uint4*>(at + c.x);
      b = *reinterpret_cast<const uint4*>(at + c.y);
    };
    if (live) fetch(h, u2, v2);
    for (; h < end; h += NW) {
      u = u2;
      v = v2;
      if (live && h + NW < end) fetch(h + NW, u2, v2);
      if (norm) do_row<D, PAIRS, true>(u, v, wt, cs, turn && rotated, s.eps);
      else if (turn) do_row<D, PAIRS, false>(u, v, wt, cs, rotated, s.eps);
      if (live) {
        uint16_t* const at = y + (size_t)(h - before) * s.rows * D;
        store_through(at + c.x, u);
        store_through(at + c.y, v);
      }
    }
  };
  part(P.q, P.Q, P.q_norm, 0, s.H, s.rot > 0);
  if (h1 <= s.H) return;
  part(P.k, P.K, P.k_norm, s.H, s.Hkv, s.rot > 0);
  part(P.v, P.V, nullptr, s.H + s.Hkv, s.Hkv, false);
}

// Workgroups along the heads, up to one head a wave: as many as make 1024 in all, four a CU, since each slice forms
// the angles again.  (48 heads of d 128: 500 tokens 4.3 us, at 512 in all 4.7; 2000 tokens 10.3, at 4096 11.4; 8000 tokens
// in one slice 38, in two 40.)
inline int head_slices(int64_t groups, int heads, int waves) {
  const int64_t most = (heads + waves - 1) / waves, want = groups < 1024 ? 1024 / groups : 1;
  return (int)(want < most ? want : most);
}

}  // namespace
}  // namespace ugbs
