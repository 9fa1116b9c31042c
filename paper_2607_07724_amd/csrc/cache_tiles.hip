// Attention over the cache where a request brings many rows (pieces of prompts):
// 64 rows a tile (32 at d 256), the products of cache_attend.hip.
//
// The keys of a part are split over the waves: each wave takes all of the tile's
// rows against its own halves of pages (32 keys), with its own running maxima, sums
// and O, joined at the end, so nothing in the loop waits for another wave.  With 64
// rows per byte read, widening the bytes to bf16 costs 64 of about 500 vector
// instructions a step.  O alone takes D registers a row tile of 16, so the bytes wait in
// LDS: direct loads, 1 KiB each, land in the order in which lanes read them, without
// bank conflicts.  The values' loads go out one by one between the matrix instructions
// of S, the next keys' between the exponentials (issued in a row they would stall the
// wave).
#include "cache_attend.h"

namespace ugbs {
namespace {

// ONCE: the rows of a kv head are one tile, so a byte is read once and not kept in the caches.
template <bool ONCE>
__device__ __forceinline__ void dma16_cache(const uint8_t* base, uint32_t voff, uint32_t lds_byte_addr) {
  if constexpr (ONCE) {
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :
                 : "v"(voff), "s"(base), "s"(lds_byte_addr)
                 : "memory");
  } else {
    dma16(reinterpret_cast<const uint16_t*>(base), voff, lds_byte_addr);
  }
}

// One part: RT tiles of 16 rows against pages p0 .. p1 - 1.
template <int D, int DT, int RT, int QR, int NW, int WPE, bool ONCE>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
cache_tiles_kernel(CacheAttendParams P) {
  constexpr int L = D / 32, E = D / 64;     // loads of a half page's keys (values); 64-channel steps
  constexpr int ROWS = 16 * RT;
  constexpr int kTile = 32 * D;             // bytes of a half page's keys (values)
  constexpr int kAll = NW * 2 * kTile, kOut = NW * 16 * (D + 4) * 4;
  __shared__ __align__(16) uint8_t s_mem[kAll > kOut ? kAll : kOut];
  __shared__ float2 s_ml[NW * ROWS];
  __shared__ __align__(16) uint4 s_q[QR < RT ? (RT - QR) * 2 * E * 64 : 1];   // rows of tiles QR.., as operands
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
  const uint8_t* const tk = s_mem + w * 2 * kTile;
  const uint8_t* const tv = tk + kTile;
  const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_addr(tk)), v_lds = k_lds + kTile;
  const uint32_t off = 16 * lane;
  auto load_k = [&](int page, int j) {
    dma16_cache<ONCE>(cache + page * page_stride + j * 1024, off, k_lds + j * 1024);
  };
  auto load_v = [&](int page, int j) {
    dma16_cache<ONCE>(cache + page * page_stride + kBlock * D + j * 1024, off, v_lds + j * 1024);
  };

  Pages pages = pages_of(P, u, p0, p1, w >> 1, NW / 2);
  int l = pages.next();
  int page = l >= 0 ? pages.page(l) : 0;
  const int key_first = l >= 0 ? kBlock * pages.at(l) + 32 * half : INT32_MAX;
  if (l >= 0) {
#pragma unroll
    for (int j = 0; j < L; ++j) load_k(page, j);
  }

  int last[RT];
  bf16x8 bq[QR][2 * E];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = u.tile * ROWS + 16 * rt + c16;
    const bool ok = r < u.q * s.G;
    const int i = ok ? r / s.G : 0, h = u.kvh * s.G + (ok ? r % s.G : 0);
    last[rt] = ok ? u.kv - u.q + i : -1;
    const uint16_t* const q = P.Q + (((size_t)u.b * s.H + h) * s.rows + i) * D + 16 * g;
#pragma unroll
    for (int x = 0; x < 2 * E; ++x) {
      if (rt < QR || w == rt % NW) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (ok) v = *reinterpret_cast<const uint4*>(q + 64 * (x >> 1) + 8 * (x & 1));
        if (rt < QR) bq[rt < QR ? rt : 0][x] = as_bf16x8(v);
        else s_q[((rt - QR) * 2 * E + x) * 64 + lane] = v;
      }
    }
  }
  const int all_see = u.kv - u.q + u.tile * ROWS / s.G;   // every valid row sees the keys up to here
  if constexpr (QR < RT) __syncthreads();

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
    auto raw_k = [&](int j) { return *reinterpret_cast<const uint4*>(tk + ((j & 1) * E + (j >> 1)) * 1024 + off); };
    uint4 raw[L];
    raw[0] = raw_k(0);
    bf16x8 lq[RT][2];
#pragma unroll
    for (int j = 0; j < L; ++j) {
      if (j + 1 < L) raw[j + 1] = raw_k(j + 1);
      if ((j & 1) == 0) {
#pragma unroll
        for (int rt = QR; rt < RT; ++rt)
#pragma unroll
          for (int y = 0; y < 2; ++y) lq[rt][y] = as_bf16x8(s_q[((rt - QR) * 2 * E + 2 * (j >> 1) + y) * 64 + lane]);
      }
      __builtin_amdgcn_sched_barrier(0);
      const bf16x8 a = operand<DT>(raw[j].x, raw[j].y), b = operand<DT>(raw[j].z, raw[j].w);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        sc[rt][j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, rt < QR ? bq[rt < QR ? rt : 0][2 * (j >> 1)] : lq[rt][0], sc[rt][j & 1], 0, 0, 0);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        sc[rt][j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, rt < QR ? bq[rt < QR ? rt : 0][2 * (j >> 1) + 1] : lq[rt][1], sc[rt][j & 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      load_v(page, j);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the keys are read: their place may be filled again

    if (key0 + 31 > all_see) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key0 + 16 * kt + 4 * g + e > last[rt]) sc[rt][kt][e] = -__builtin_huge_valf();
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
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (rt * ((L + RT - 1) / RT) < L) {
        __builtin_amdgcn_sched_barrier(0);
        if (l >= 0) {
#pragma unroll
          for (int j = rt * ((L + RT - 1) / RT); j < (rt + 1) * ((L + RT - 1) / RT) && j < L; ++j) load_k(page2, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
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
    }
    __builtin_amdgcn_sched_barrier(0);
    // the values have landed; the L younger loads (the next keys) may be on their way
    if (l >= 0) wait_vmcnt<L>();
    else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    if (key0 + 32 > u.kv) {                              // each lane's own 16 bytes of each load
      const uint2 keep = live_bytes(u.kv, key0);
#pragma unroll
      for (int j = 0; j < L; ++j) {
        uint4* const x = reinterpret_cast<uint4*>(s_mem + w * 2 * kTile + kTile + j * 1024 + off);
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
  for (int rt = 0; rt < RT; ++rt) seen[rt] = key_first <= last[rt];
  __syncthreads();                                       // the waves' tiles make room for the sums
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
