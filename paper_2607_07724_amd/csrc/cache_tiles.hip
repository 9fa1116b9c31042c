// Attention over the cache where a request brings many rows (pieces of prompts):
// 64 rows a tile (32 at d 256), the products of cache_attend.hip.
//
// The keys of a part are split over the waves: each wave takes all of the tile's
// rows against its own halves of pages (32 keys), with its own running maxima, sums
// and O, joined at the end, so nothing in the loop waits for another wave.  e4m3
// keys of 128 or 256 channels are operands as they are (see split_row); the values, and
// all other bytes, are widened to bf16 once for the 64 rows.  Bound by the vector unit
// (exponentials, widening) beside the matrix cores: two pieces of 1024 tokens on up to 33K
// (32/8 heads, d 128) 608-657 us, 1.07-1.16 PFLOP/s.
// O alone takes D registers a row tile of 16, so the bytes wait in LDS: direct loads,
// 1 KiB each, land in the order in which lanes read them, without bank conflicts.  The
// values' loads go out one by one between the matrix instructions of S, the next keys'
// between the exponentials (issued in a row they would stall the wave).
#include <type_traits>

#include "cache_attend.h"

namespace ugbs {
namespace {

// ONCE: the rows of a kv head are one tile, so a byte is read once and not kept in the caches.
// The offset counts for both sides: base + voff + OFF to the lane's 16 bytes at lds + OFF.
template <bool ONCE, int OFF>
__device__ __forceinline__ void dma16_cache(const uint8_t* base, uint32_t voff, uint32_t lds_byte_addr) {
  static_assert(OFF >= 0 && OFF < 4096, "signed 13-bit offset");
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 offset:%3 nt"
                 :
                 : "v"(voff), "s"(base), "s"(lds_byte_addr), "n"(OFF)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 offset:%3"
                 :
                 : "v"(voff), "s"(base), "s"(lds_byte_addr), "n"(OFF)
                 : "memory");
}

// f(0) .. f(N - 1) with indexes that are constants
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ i32x8 join(uint4 a, uint4 b) {
  return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// This lane's 32 channels of a 128-channel step of a row (16 g + 0..15 of each 64; 4 times 8
// bf16) to e4m3 pairs, [hi, lo][64][16 channels].  32 channels in a row share a scale: those of
// lane groups 2 j and 2 j + 1 of the first 64 (j), and of the second (2 + j), whose exponent
// the instruction takes from lane group j, or 2 + j.  Returns the lane's exponent of hi's
// scale (lo's is 5 less).
__device__ __forceinline__ uint32_t split_row(uint4* v) {
  const int g = (threadIdx.x & 63) >> 4;
  int ex[2];
  uint4 out[4];
#pragma unroll
  for (int x = 0; x < 2; ++x) {                          // 16 channels: two of the eights
    uint32_t a = 0;
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const uint4 from = v[2 * x + y / 4];
      const uint32_t w = y % 4 == 0 ? from.x : y % 4 == 1 ? from.y : y % 4 == 2 ? from.z : from.w;
      a = max(a, max(w << 16 & 0x7fffffffu, w & 0x7fff0000u));
    }
    const auto pair = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    a = max((uint32_t)pair[0], (uint32_t)pair[1]);       // with lane group g ^ 1
    ex[x] = max((int)(a >> 23) - 7, 27);                 // the largest becomes 128..255
    const float inv = __uint_as_float((uint32_t)(254 - ex[x]) << 23);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {                        // 4 channels
      const uint4 from = v[2 * x + y / 2];
      const uint32_t w0 = y % 2 ? from.z : from.x, w1 = y % 2 ? from.w : from.y;
      const float c[4] = {__uint_as_float(w0 << 16) * inv, __uint_as_float(w0 & 0xffff0000u) * inv,
                          __uint_as_float(w1 << 16) * inv, __uint_as_float(w1 & 0xffff0000u) * inv};
      int h = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
      h = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], h, true);
      const float r[4] = {(c[0] - __builtin_amdgcn_cvt_f32_fp8(h, 0)) * 32.0f, (c[1] - __builtin_amdgcn_cvt_f32_fp8(h, 1)) * 32.0f,
                          (c[2] - __builtin_amdgcn_cvt_f32_fp8(h, 2)) * 32.0f, (c[3] - __builtin_amdgcn_cvt_f32_fp8(h, 3)) * 32.0f};
      int l = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
      l = __builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], l, true);
      hi[y] = (uint32_t)h;
      lo[y] = (uint32_t)l;
    }
    out[x] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    out[2 + x] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) v[x] = out[x];
  const int far0 = __shfl_xor(ex[0], 32), far1 = __shfl_xor(ex[1], 32);
  return (uint32_t)(g == 0 ? ex[0] : g == 1 ? far0 : g == 2 ? far1 : ex[1]);
}

// One part: RT tiles of 16 rows against pages p0 .. p1 - 1.
template <int D, int DT, int RT, int QR, int NW, int WPE, bool ONCE>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
cache_tiles_kernel(CacheAttendParams P) {
  constexpr int L = D / 32, E = D / 64;     // loads of a half page's keys (values); 64-channel steps
  constexpr int ROWS = 16 * RT;
  constexpr bool F8 = DT == UGBS_E4M3 && D >= 128;
  constexpr int kTile = 32 * D;             // bytes of a half page's keys (values)
  __shared__ __align__(16) uint8_t s_mem[NW * 2 * kTile];   // at the end: 16 rows' sums of every wave
  static_assert(sizeof(float) * NW * 16 * D <= NW * 2 * kTile, "they fit");
  __shared__ float2 s_ml[NW * ROWS];
  __shared__ __align__(16) uint4 s_q[QR < RT ? (RT - QR) * 2 * E * 64 : 1];   // rows of tiles QR.., as operands
  __shared__ uint32_t s_qs[F8 ? RT * (E / 2) * 64 : 1];                                     // their scales
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
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

  const int half = w & 1;
  const uint8_t* const cache = P.cache + (size_t)u.kvh * 2 * (kBlock * D) + half * kTile;
  const size_t page_stride = (size_t)s.Hkv * 2 * (kBlock * D);
  uint8_t* const tk = s_mem + w * 2 * kTile;
  uint8_t* const tv = tk + kTile;
  const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_addr(tk)), v_lds = k_lds + kTile;
  const uint32_t off = 16 * lane;
  auto keys_of = [&](int page) { return cache + page * page_stride; };
  auto load_k = [&](const uint8_t* src, auto j) {
    dma16_cache<ONCE, j % 4 * 1024>(src + j / 4 * 4096, off, k_lds + j / 4 * 4096);
  };
  auto load_v = [&](const uint8_t* src, auto j) {
    dma16_cache<ONCE, j % 4 * 1024>(src + kBlock * D + j / 4 * 4096, off, v_lds + j / 4 * 4096);
  };

  Pages pages = pages_of(P, u, p0, p1, w >> 1, NW / 2);
  int l = pages.next();
  int page = l >= 0 ? pages.page(l) : 0;
  const int key_first = l >= 0 ? kBlock * pages.at(l) + 32 * half : INT32_MAX;
  if (l >= 0) each<L>([&](auto j) { load_k(keys_of(page), j); });

  // The rows as the B operand.  F8: each channel is split into two e4m3 numbers, which
  // with a power of two for each 32 channels of a row, the instruction's own scales, give
  // the bf16 number back: the largest of the 32 is brought to 128..255, hi is a number's
  // nearest with 4 significant bits, and what is left has at most 4.  (Numbers below 2^-13
  // of the largest of their 32, taken as 2^-93 at least, lose what lies below 2^-22 of it.)
  // So the keys' bytes are operands as they are; on this instruction two such products cost
  // what one in bf16 does (pieces of 1024 tokens, d 128: 645 -> 611 us, d 256: 724 -> 668).
  uint4 bq[QR][2 * E];                      // F8: [E / 2][hi, lo][2], 16 channels each
  constexpr int C = F8 ? E / 2 : 1;         // 128-channel steps
  uint32_t q_hi[C] = {}, q_lo[C];           // F8: exponents (E8M0) of row tile rt's hi and lo in byte rt
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = u.tile * ROWS + 16 * rt + c16;
    const bool ok = r < u.q * s.G;
    const int i = ok ? r / s.G : 0, h = u.kvh * s.G + (ok ? r % s.G : 0);
    if (F8 ? w == rt : rt < QR || w == rt % NW) {
      const uint16_t* const q = P.Q + (((size_t)u.b * s.H + h) * s.rows + i) * D + 16 * g;
      uint4 v[2 * E];
#pragma unroll
      for (int x = 0; x < 2 * E; ++x) {
        v[x] = make_uint4(0, 0, 0, 0);
        if (ok) v[x] = *reinterpret_cast<const uint4*>(q + 64 * (x >> 1) + 8 * (x & 1));
      }
      if constexpr (F8) {
#pragma unroll
        for (int c = 0; c < C; ++c) s_qs[(rt * C + c) * 64 + lane] = split_row(v + 4 * c) << 8 * rt;
      }
      // F8: one wave splits a row tile; those that go to registers pass through its values' place
      uint4* const to = rt < QR ? reinterpret_cast<uint4*>(tv) : s_q + (rt - QR) * 2 * E * 64;
#pragma unroll
      for (int x = 0; x < 2 * E; ++x) {
        if (!F8 && rt < QR) bq[rt < QR ? rt : 0][x] = v[x];
        else to[x * 64 + lane] = v[x];
      }
    }
  }
  if constexpr (QR < RT || F8) __syncthreads();
  if constexpr (F8) {
    static_assert(RT <= NW && 2 * E * 1024 <= kTile, "a row tile to a wave, in the place of its values");
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) q_hi[c] |= s_qs[(rt * C + c) * 64 + lane];
      q_lo[c] = q_hi[c] - 0x05050505u;      // (exponents are 27 at least)
    }
#pragma unroll
    for (int rt = 0; rt < QR; ++rt)
#pragma unroll
      for (int x = 0; x < 2 * E; ++x) bq[rt][x] = reinterpret_cast<const uint4*>(s_mem + rt * 2 * kTile + kTile)[x * 64 + lane];
    __syncthreads();
  }

  // the last key that the lane's row in tile rt sees (asked for at the ends of requests only)
  auto last = [&](int rt) {
    const int r = u.tile * ROWS + 16 * rt + (int)here(c16);
    return r < u.q * s.G ? u.kv - u.q + r / s.G : -1;
  };
  const int all_see = u.kv - u.q + u.tile * ROWS / s.G;   // every valid row sees the keys up to here

  f32x4 acc[RT][D / 16];
  float m_run[RT], l_run[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[rt] = kNoMax;
    l_run[rt] = 0.f;
  }

  while (l >= 0) {
    const int key0 = kBlock * pages.at(l) + 32 * half;
    // (a factor that underflows would make masked scores NaN)
    const float f = fmaxf(pages.key_scale(l) * P.scale_log2, 1.17549435e-38f), vs = pages.value_scale(l);
    l = pages.next();
    const int page2 = l >= 0 ? pages.page(l) : 0;
    wait_vmcnt<0>();                                     // the keys have landed
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_setprio(0);
    // ---- S^T; the values' loads go out between the matrix instructions
    f32x4 sc[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sc[rt][0] = sc[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint8_t* const src = keys_of(page);
    auto raw_k = [&](int kt, int e) { return *reinterpret_cast<const uint4*>(tk + (kt * E + e) * 1024 + off); };
    auto row_at = [&](int rt, int x) { return rt < QR ? bq[rt < QR ? rt : 0][x] : s_q[((rt - QR) * 2 * E + x) * 64 + lane]; };
    if constexpr (F8) {
      // 16 keys x 128 channels an instruction; (kt, c) = (j % 2, j / 2).  The rows that are
      // in registers first, the others' parts (8 registers each) read two ahead.
      uint4 raw[2][2];
      raw[0][0] = raw_k(0, 0);
      raw[0][1] = raw_k(0, 1);
      each<E>([&](auto j) {
        constexpr int kt = j % 2, c = j / 2, NL = 2 * (RT - QR);
        uint4 lq[NL > 0 ? NL : 1][2];
        auto read = [&](auto x) {           // part x: hi of the rows in LDS, then lo
          constexpr int rt = QR + x % (RT - QR), part = x / (RT - QR);
#pragma unroll
          for (int y = 0; y < 2; ++y) lq[x][y] = row_at(rt, 4 * c + 2 * part + y);
        };
        auto mul = [&](auto rt, auto part, uint4 q0, uint4 q1) {
          sc[rt][kt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(join(raw[j % 2][0], raw[j % 2][1]), join(q0, q1), sc[rt][kt], 0, 0, 0,
                                                                        127, rt, part == 0 ? q_hi[c] : q_lo[c]);
        };
        if constexpr (NL > 0) each<(NL < 2 ? NL : 2)>(read);
        __builtin_amdgcn_sched_barrier(0);
        each<2 * QR>([&](auto x) {
          constexpr int rt = x % QR, part = x / QR;
          mul(std::integral_constant<int, rt>{}, std::integral_constant<int, part>{}, bq[rt][4 * c + 2 * part], bq[rt][4 * c + 2 * part + 1]);
        });
        __builtin_amdgcn_sched_barrier(0);
        load_v(src, std::integral_constant<int, 2 * j>{});
        if constexpr (NL > 0) {
          each<NL>([&](auto x) {
            constexpr int rt = QR + x % (RT - QR), part = x / (RT - QR);
            mul(std::integral_constant<int, rt>{}, std::integral_constant<int, part>{}, lq[x][0], lq[x][1]);
            if constexpr (x + 2 < NL) read(std::integral_constant<int, x + 2>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        }
        if constexpr (j + 1 < E) {
          raw[(j + 1) % 2][0] = raw_k((j + 1) % 2, (j + 1) / 2 * 2);
          raw[(j + 1) % 2][1] = raw_k((j + 1) % 2, (j + 1) / 2 * 2 + 1);
        }
        load_v(src, std::integral_constant<int, 2 * j + 1>{});
      });
    } else {
      uint4 raw[L];
      raw[0] = raw_k(0, 0);
      uint4 lq[RT][2];
      each<L>([&](auto j) {
        constexpr int kt = j % 2, e = j / 2;
        if constexpr (j + 1 < L) raw[j + 1] = raw_k((j + 1) % 2, (j + 1) / 2);
        if constexpr (kt == 0) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int y = 0; y < 2; ++y) lq[rt][y] = row_at(rt, 2 * e + y);
        }
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 a = operand<DT>(raw[j].x, raw[j].y), b = operand<DT>(raw[j].z, raw[j].w);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(lq[rt][0]), sc[rt][kt], 0, 0, 0);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, as_bf16x8(lq[rt][1]), sc[rt][kt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_v(src, j);
      });
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the keys are read: their place may be filled again

    if (key0 + 31 > all_see) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int end = last(rt);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key0 + 16 * kt + 4 * g + e > end) sc[rt][kt][e] = -__builtin_huge_valf();
      }
    }
    // ---- softmax: the maximum only moves when a score exceeds it by more than 2^8 (asked per lane first)
    float mx[RT], over = -__builtin_huge_valf();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const f32x4 a = sc[rt][0], b = sc[rt][1];
      float m = fmaxf(fmaxf(a[0], a[1]), a[2]);
      m = fmaxf(fmaxf(m, a[3]), b[0]);
      m = fmaxf(fmaxf(m, b[1]), b[2]);
      mx[rt] = fmaxf(m, b[3]);
      over = fmaxf(over, __builtin_fmaf(mx[rt], f, -m_run[rt]));
    }
    if (__ballot(over > 8.0f)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float r = rows_max(mx[rt]) * f;
        const float m_new = r > m_run[rt] + 8.0f ? r : m_run[rt];
        const float alpha = r > m_run[rt] + 8.0f ? __builtin_amdgcn_exp2f(m_run[rt] - m_new) : 1.0f;
        m_run[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[rt][dt][e] *= alpha;
      }
    }
    uint32_t pb[RT][4];
    const uint8_t* const src2 = keys_of(page2);
    each<RT>([&](auto rt) {
      constexpr int n = (L + RT - 1) / RT, first = rt * n;      // the next keys' loads
      __builtin_amdgcn_sched_barrier(0);
      if (l >= 0) each<(first + n <= L ? n : L - first)>([&](auto j) { load_k(src2, std::integral_constant<int, first + j>{}); });
      __builtin_amdgcn_sched_barrier(0);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rt][e >> 2][e & 3], f, -m_run[rt]));
        l_run[rt] += p[e];
        if (DT != UGBS_E4M3) p[e] *= vs;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) pb[rt][e] = pack_bf16(p[2 * e], p[2 * e + 1]);
      // the softmax is complete here (else its ends are moved behind the wait and hold registers over PV)
      asm volatile("" : "+v"(l_run[rt]), "+v"(pb[rt][0]), "+v"(pb[rt][1]), "+v"(pb[rt][2]), "+v"(pb[rt][3]));
    });
    __builtin_amdgcn_sched_barrier(0);
    // the values have landed; the L younger loads (the next keys) may be on their way
    if (l >= 0) wait_vmcnt<L>();
    else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    if (key0 + 32 > u.kv) {                              // each lane's own 16 bytes of each load
      const uint2 keep = live_bytes(u.kv, key0);
#pragma unroll
      for (int j = 0; j < L; ++j) {
        uint4* const x = reinterpret_cast<uint4*>(tv + j * 1024 + off);
        const uint4 y = *x;
        *x = make_uint4(y.x & keep.x, y.y & keep.y, y.z & keep.x, y.w & keep.y);
      }
    }
    // ---- O^T += V^T P^T
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const uint4 x = *reinterpret_cast<const uint4*>(tv + j * 1024 + off);
      const bf16x8 a = operand<DT>(x.x, x.y, vs), b = operand<DT>(x.z, x.w, vs);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const bf16x8 bp = as_bf16x8(make_uint4(pb[rt][0], pb[rt][1], pb[rt][2], pb[rt][3]));
        acc[rt][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bp, acc[rt][2 * j], 0, 0, 0);
        acc[rt][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, bp, acc[rt][2 * j + 1], 0, 0, 0);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the values are read
    page = page2;
  }

  bool seen[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) seen[rt] = key_first <= last(rt);
  finish_part<D, RT, NW>(P, u, reinterpret_cast<float*>(s_mem), s_ml, acc, m_run, l_run, seen);
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
