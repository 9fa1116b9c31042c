// Attention of a batch whose requests list common first pages: these pages once for all rows of
// a group, the pages that are a request's own for its rows, and the join of both.
//
// A softmax over the keys of pages P u R is what the two sets give apart: with M, l and o the
// maximum, the sum and the weighted values of each, the result is
//   (2^(M_P - M) o_P + 2^(M_R - M) o_R) / (2^(M_P - M) l_P + 2^(M_R - M) l_R),  M = max(M_P, M_R),
// the join that parts along the pages need anyway.  What is won is bytes: a page of the prefix
// is read once for up to 64 rows of a kv head, of all requests of the group, instead of once for each request.
//
// ugbs_cache_share finds, once a step, what the requests of a group have in common (their table
// rows are compared, so nothing but the table says what is shared) and lays the parts out,
// as ugbs_cache_attend does for itself; the launches of a layer only look their part up.
#include "cache_attend.h"

namespace ugbs {
namespace {

// A group shares its common pages from this many saved page reads of a kv head on.
constexpr int kLeastSaved = 1;
// More query rows to a kv head than this fill a tile by themselves.
constexpr int kMostRows = 64;

// (the join's grid: a workgroup for each row)
bool shares(const CacheShape& s) {
  return s.B > 1 && (int64_t)s.rows * s.G <= kMostRows && (int64_t)s.B * s.rows * s.H <= (1 << 20);
}

struct Sizes {
  int own_rows, prefix_rows;          // of a tile
  int64_t own_parts, prefix_parts;    // at most
  int64_t sum_rows;                   // rows of the parts' sums, at most
};

// A part more than the tiles for each of kTarget at most; a group has two requests at least.
Sizes sizes_of(const CacheShape& s) {
  const int64_t all = (int64_t)s.B * s.rows * s.G, groups = s.B / 2;
  Sizes z;
  z.own_rows = tile_rows(s);
  z.prefix_rows = tile_rows(s.d, all);
  z.own_parts = tiles_bound(s, z.own_rows) + kTarget;
  z.prefix_parts = s.Hkv * (all / z.prefix_rows + groups) + kTarget;
  z.sum_rows = s.Hkv * (s.B * (((int64_t)s.rows * s.G + 15) / 16 * 16) + all + 15 * groups) + kTarget * (z.own_rows + z.prefix_rows);
  return z;
}

// The arrays of a plan, one behind another; returns their bytes.
size_t lay_out(const CacheShape& s, void* at, Share* share) {
  const Sizes z = sizes_of(s);
  uint8_t* const base = static_cast<uint8_t*>(at);
  size_t n = 0;
  auto take = [&](size_t bytes) {
    uint8_t* const p = base + n;
    n += align256(bytes);
    return p;
  };
  share->own = reinterpret_cast<int4*>(take(3 * sizeof(int4) * s.B));
  share->prefix = reinterpret_cast<int4*>(take(2 * sizeof(int4) * s.B));
  share->own_part = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * z.own_parts));
  share->prefix_part = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * z.prefix_parts));
  share->row = reinterpret_cast<int2*>(take(sizeof(int2) * s.B * s.rows));
  share->found = reinterpret_cast<int4*>(take(sizeof(int4) * s.B));
  return n;
}

// What request b (a workgroup) has in common with the first request of its group: whole pages, full
// for both, whose entries are the same from the first on.
__global__ void __launch_bounds__(256) share_compare_kernel(CacheAttendParams P, const int32_t* __restrict__ group) {
  __shared__ int s_min[4], s_before[4], s_members[4], s_differs[4];
  const int b = blockIdx.x, tid = threadIdx.x, w = tid >> 6, mine = group[b];
  const int q = min(max(P.q_lens[b], 0), P.s.rows);
  if (mine < 0 || q == 0) {
    if (tid == 0) P.share.found[b] = make_int4(-1, 0, 0, 0);
    return;
  }
  int leader = INT32_MAX, before = 0, members = 0;
  for (int x = tid; x < P.s.B; x += 256) {
    const int n = min(max(P.q_lens[x], 0), P.s.rows);
    if (group[x] == mine && n > 0) {
      leader = min(leader, x);
      if (x < b) before += n;
      ++members;
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    leader = min(leader, __shfl_xor(leader, o));
    before += __shfl_xor(before, o);
    members += __shfl_xor(members, o);
  }
  if ((tid & 63) == 0) {
    s_min[w] = leader;
    s_before[w] = before;
    s_members[w] = members;
  }
  __syncthreads();
  leader = min(min(s_min[0], s_min[1]), min(s_min[2], s_min[3]));
  before = s_before[0] + s_before[1] + s_before[2] + s_before[3];
  members = s_members[0] + s_members[1] + s_members[2] + s_members[3];
  const int most = P.s.max_pages * kBlock;
  const int full = min(min(max(P.kv_lens[b], 0), most), min(max(P.kv_lens[leader], 0), most)) / kBlock;
  const int32_t* const x = P.table + (size_t)b * P.s.max_pages;
  const int32_t* const y = P.table + (size_t)leader * P.s.max_pages;
  int differs = full;
  if (b != leader)
    for (int j = tid; j < differs; j += 256)
      if (x[j] != y[j]) differs = j;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) differs = min(differs, __shfl_xor(differs, o));
  if ((tid & 63) == 0) s_differs[w] = differs;
  __syncthreads();
  if (tid == 0) {
    differs = min(min(s_differs[0], s_differs[1]), min(s_differs[2], s_differs[3]));
    P.share.found[b] = make_int4(members > 1 ? leader : -1, differs, before, 0);
  }
}

// Sums over the workgroup, before this thread and in all.
constexpr int kPlanThreads = 1024, kPer = UGBS_MAX_REQUESTS / kPlanThreads;
__device__ __forceinline__ float sum_all(float x, float* s_wave) {
  x = sum_wave(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int v = 0; v < kPlanThreads / 64; ++v) x += s_wave[v];
  return x;
}
__device__ __forceinline__ int sum_before(int x, int* s_wave, int* total) {
  const int upto = scan_add(x), w = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s_wave[w] = upto;
  __syncthreads();
  int before = upto - x;
  *total = 0;
#pragma unroll
  for (int v = 0; v < kPlanThreads / 64; ++v) {
    if (v < w) before += s_wave[v];
    *total += s_wave[v];
  }
  return before;
}

// The parts.  Every workgroup forms the sums over all requests (4 a thread); the first one writes
// the requests' entries, all write their share of the lists.
__global__ void __launch_bounds__(kPlanThreads) share_plan_kernel(CacheAttendParams P, int own_rows, int prefix_rows, int own_parts,
                                                                  int prefix_parts) {
  __shared__ int s_a[UGBS_MAX_REQUESTS], s_b[UGBS_MAX_REQUESTS], s_c[UGBS_MAX_REQUESTS];
  __shared__ float s_sum[kPlanThreads / 64];
  __shared__ int s_scan[kPlanThreads / 64];
  const int tid = threadIdx.x, B = P.s.B, G = P.s.G, Hkv = P.s.Hkv, most = P.s.max_pages * kBlock;
  for (int b = tid; b < B; b += kPlanThreads) {
    s_a[b] = INT32_MAX;
    s_b[b] = s_c[b] = 0;
  }
  __syncthreads();
  int4 found[kPer];
  Lengths own[kPer], pre[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = kPer * tid + k;
    found[k] = make_int4(-1, 0, 0, 0);
    own[k] = pre[k] = Lengths{0, 0, 0, 0};
    if (b >= B) continue;
    found[k] = P.share.found[b];
    own[k].q = min(max(P.q_lens[b], 0), P.s.rows);
    own[k].kv = min(max(P.kv_lens[b], 0), most);
    const int l = found[k].x;
    if (l >= 0) {
      atomicMin(&s_a[l], found[k].y);                          // pages in common
      atomicMax(&s_b[l], found[k].z + own[k].q);               // new tokens
      atomicAdd(&s_c[l], 1);
    }
  }
  __syncthreads();
  int together[kPer];                                          // new tokens of the group, 0: nothing is shared
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = kPer * tid + k, l = found[k].x;
    together[k] = 0;
    int pages = 0;
    if (l >= 0 && s_a[l] * (s_c[l] - 1) >= kLeastSaved) {
      pages = s_a[l];
      together[k] = s_b[l];
    }
    found[k].y = pages;
    own[k].tiles = (own[k].q * G + own_rows - 1) / own_rows;
    own[k].pages = max((own[k].kv + kBlock - 1) / kBlock - pages, 0);
    if (pages > 0 && b == l) {
      pre[k].q = together[k];
      pre[k].tiles = (together[k] * G + prefix_rows - 1) / prefix_rows;
      pre[k].pages = pages;
    }
  }
  auto per_part = [&](const Lengths (&r)[kPer], int rows) {
    float work = 0.f, tiles = 0.f, wide = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      work = __builtin_fmaf((float)r[k].tiles, (float)r[k].pages, work);
      tiles += (float)r[k].tiles;
    }
    work = sum_all(work, s_sum);
    tiles = sum_all(tiles, s_sum);
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (is_wide(P, r[k], work)) wide += (float)r[k].tiles;
    return pages_per_part(P, rows, work, tiles, sum_all(wide, s_sum));
  };
  const int per_own = per_part(own, own_rows), per_pre = per_part(pre, prefix_rows);
  // parts and rows of sums of the requests and of the groups, and the groups' new tokens
  int n[5] = {0, 0, 0, 0, 0}, at[5], total[5];
  auto count = [&](int k, int (&x)[5]) {
    const int so = splits_of(own[k], per_own), sp = splits_of(pre[k], per_pre);
    x[0] = own[k].tiles * Hkv * so;
    x[1] = own[k].tiles > 0 && (so > 1 || found[k].y > 0) ? so * Hkv * ((own[k].q * G + 15) / 16 * 16) : 0;
    x[2] = pre[k].tiles * Hkv * sp;
    x[3] = sp * Hkv * ((pre[k].q * G + 15) / 16 * 16);
    x[4] = pre[k].q;
  };
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    int x[5];
    count(k, x);
#pragma unroll
    for (int y = 0; y < 5; ++y) n[y] += x[y];
  }
#pragma unroll
  for (int y = 0; y < 5; ++y) at[y] = sum_before(n[y], s_scan, &total[y]);
  at[3] += total[1];                                           // behind the requests' own
  // (the barriers of the sums are behind the last reads of s_a .. s_c)
  int first[kPer][5];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = kPer * tid + k;
    int x[5];
    count(k, x);
#pragma unroll
    for (int y = 0; y < 5; ++y) {
      first[k][y] = at[y];
      at[y] += x[y];
    }
    if (b < B && pre[k].tiles > 0) {
      s_a[b] = first[k][3];
      s_b[b] = splits_of(pre[k], per_pre);
      s_c[b] = first[k][4];
    }
  }
  __syncthreads();
  if (blockIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int b = kPer * tid + k, l = found[k].x, so = splits_of(own[k], per_own), pages = found[k].y;
      if (b >= B) continue;
      int4* const o = P.share.own + 3 * b;
      o[0] = make_int4(first[k][0], so, so > 1 || pages > 0 ? first[k][1] : -1, pages);
      o[1] = pages > 0 ? make_int4(s_a[l], s_b[l], found[k].z, (together[k] * G + 15) / 16 * 16) : make_int4(-1, 0, 0, 0);
      o[2] = make_int4(own[k].q, own[k].kv, 0, 0);
      P.share.prefix[2 * b] = make_int4(first[k][2], splits_of(pre[k], per_pre), first[k][3], first[k][4]);
      P.share.prefix[2 * b + 1] = make_int4(pre[k].q, pre[k].pages, 0, 0);
      if (pages > 0)
        for (int i = 0; i < own[k].q; ++i)
          P.share.row[s_c[l] + found[k].z + i] = make_int2(b * P.s.rows + i, own[k].kv - own[k].q + i);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = kPer * tid + k;
    if (b < B) {
      s_a[b] = first[k][0];
      s_b[b] = first[k][2];
    }
  }
  __syncthreads();
  // the last request with sums[b] <= i (those without parts have the same sum as the next)
  auto request_at = [&](const int* sums, int i) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (sums[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  const int stride = gridDim.x * kPlanThreads;
  for (int i = blockIdx.x * kPlanThreads + tid; i < own_parts; i += stride) P.share.own_part[i] = i < total[0] ? request_at(s_a, i) : -1;
  for (int i = blockIdx.x * kPlanThreads + tid; i < prefix_parts; i += stride)
    P.share.prefix_part[i] = i < total[2] ? request_at(s_b, i) : -1;
}

// Joins the parts of the rows of a request, those of the prefix first: NT threads to a row, D / 4 to a
// part of it, eight parts of a thread on their way at once.
template <int D, int NT>
__global__ void __launch_bounds__(256) share_join_kernel(CacheAttendParams P, int own_rows, int prefix_rows) {
  constexpr int CG = D / 4, GR = NT / CG, ROWS = 256 / NT, W = NT / 64, kAhead = 8;
  constexpr int kMost = 2 * (kTarget + 1);  // parts of a row
  __shared__ float s_weight[ROWS][kMost];
  __shared__ float2 s_ml[4];
  __shared__ f32x4 s_o[W > 1 ? GR : 1][CG];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, G = P.s.G;
  const int b = blockIdx.x / P.s.Hkv, kvh = blockIdx.x % P.s.Hkv, mine = tid / NT, t = tid % NT;
  const int r = blockIdx.y * ROWS + mine;
  const int4 x = P.share.own[3 * b], y = P.share.own[3 * b + 1], z = P.share.own[3 * b + 2];
  // (a row's threads leave together: no barrier where there is a wave or less to a row)
  if (x.z < 0 || r >= z.x * G) return;
  const int all = (z.x * G + 15) / 16 * 16, tile = r / own_rows;
  const int64_t own = (int64_t)x.z + (int64_t)x.y * (kvh * all + tile * own_rows) + r % own_rows;
  const int step = min(own_rows, all - tile * own_rows), np = y.x < 0 ? 0 : y.y;
  const int rp = y.z * G + r, tp = rp / prefix_rows;
  const int64_t prefix = (int64_t)y.x + (int64_t)np * (kvh * y.w + tp * prefix_rows) + rp % prefix_rows;
  const int step_p = min(prefix_rows, y.w - tp * prefix_rows), parts = min(np + x.y, kMost);
  auto at = [&](int v) { return v < np ? prefix + (int64_t)v * step_p : own + (int64_t)(v - np) * step; };
  float M = -__builtin_huge_valf();
  for (int v = t; v < parts; v += NT) M = fmaxf(M, P.part_ml[at(v)].x);
  const int gr = t / CG, c = t % CG;
  const f32x4* const po = reinterpret_cast<const f32x4*>(P.part_o) + c;
  f32x4 ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (k * GR < parts) ahead[k] = po[at(min(gr + k * GR, parts - 1)) * CG];
#pragma unroll
  for (int o = 1; o < 64; o *= 2) M = fmaxf(M, __shfl_xor(M, o));
  if constexpr (W > 1) {
    if (lane == 0) s_ml[w].x = M;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < W; ++v) M = fmaxf(M, s_ml[v].x);
  }
  float l = 0.f;
  for (int v = t; v < parts; v += NT) {
    const float2 m = P.part_ml[at(v)];
    const float a = m.x == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(m.x - M);   // it saw none of the row's keys
    s_weight[mine][v] = a;
    if (a != 0.f) l += a * m.y;
  }
  l = sum_wave(l);
  if constexpr (W > 1) {
    if (lane == 0) s_ml[w].y = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int v = 0; v < W; ++v) l += s_ml[v].y;
  } else {
    // the weights are read by other lanes of the wave that wrote them
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](int v, const f32x4& p) {
    const float a = s_weight[mine][v];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += a * p[e];
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (gr + k * GR < parts) add(gr + k * GR, ahead[k]);
  for (int v0 = kAhead * GR; v0 < parts; v0 += kAhead * GR) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v0 + k * GR < parts) ahead[k] = po[at(min(v0 + gr + k * GR, parts - 1)) * CG];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v0 + gr + k * GR < parts) add(v0 + gr + k * GR, ahead[k]);
  }
  if constexpr (W > 1) {
    s_o[gr][c] = o;
    __syncthreads();
    if (gr > 0) return;
#pragma unroll
    for (int v = 1; v < GR; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += s_o[v][c][e];
  } else {
#pragma unroll
    for (int s = CG; s < 64; s *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], s);
    if (gr > 0) return;
  }
  Part u;
  u.b = b;
  u.kvh = kvh;
  store_row(P, u, D, r, 4 * c, o, reciprocal(M, l));
}

template <int D>
void join_shared(const CacheAttendParams& P, const Sizes& z, hipStream_t stream) {
  const int rows = P.s.rows * P.s.G;
  share_join_kernel<D, 256><<<dim3((unsigned)(P.s.B * P.s.Hkv), rows), 256, 0, stream>>>(P, z.own_rows, z.prefix_rows);
}

CacheAttendParams params_of(const CacheShape& s, const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens) {
  CacheAttendParams P{};
  P.s = s;
  P.table = table;
  P.kv_lens = kv_lens;
  P.q_lens = q_lens;
  P.scale_log2 = s.scale * 1.4426950408889634f;
  P.splits = may_split(s);
  P.min_pages = min_pages(s.d);
  return P;
}

}  // namespace

size_t cache_share_bytes(const CacheShape& s) {
  Share share;
  return shares(s) ? lay_out(s, nullptr, &share) : 256;
}

size_t cache_shared_workspace(const CacheShape& s) {
  return shares(s) ? (size_t)sizes_of(s).sum_rows * (s.d * sizeof(float) + sizeof(float2)) : cache_attend_workspace(s);
}

hipError_t launch_cache_share(const CacheShape& s, const int32_t* group, const int32_t* table, const int32_t* kv_lens,
                              const int32_t* q_lens, void* share, hipStream_t stream) {
  if (!shares(s)) return hipSuccess;
  CacheAttendParams P = params_of(s, table, kv_lens, q_lens);
  lay_out(s, share, &P.share);
  const Sizes z = sizes_of(s);
  share_compare_kernel<<<(unsigned)s.B, 256, 0, stream>>>(P, group);
  const int64_t want = (z.own_parts + z.prefix_parts + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  share_plan_kernel<<<(unsigned)(want < 64 ? want : 64), kPlanThreads, 0, stream>>>(P, z.own_rows, z.prefix_rows, (int)z.own_parts,
                                                                                  (int)z.prefix_parts);
  return hipGetLastError();
}

hipError_t launch_cache_attend_shared(const CacheShape& s, const uint16_t* Q, const uint8_t* cache, const float* scales,
                                      const int32_t* table, const int32_t* kv_lens, const int32_t* q_lens, const void* share,
                                      uint16_t* O, void* workspace, hipStream_t stream) {
  if (!shares(s)) return launch_cache_attend(s, Q, cache, scales, table, kv_lens, q_lens, O, workspace, stream);
  CacheAttendParams P = params_of(s, table, kv_lens, q_lens);
  P.Q = Q;
  P.cache = cache;
  P.scales = scales;
  P.O = O;
  lay_out(s, const_cast<void*>(share), &P.share);
  const Sizes z = sizes_of(s);
  P.part_o = static_cast<float*>(workspace);
  P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)z.sum_rows * s.d);
  auto parts = [&](Mode mode, int rows, int64_t n, bool once) {
    if (rows == tile_rows_many(s.d)) launch_shared_tiles(P, mode, (unsigned)n, once, stream);
    else launch_shared_rows(P, mode, (unsigned)n, rows, stream);
  };
  parts(kPrefix, z.prefix_rows, z.prefix_parts, (int64_t)s.B * s.rows * s.G <= z.prefix_rows);
  parts(kOwn, z.own_rows, z.own_parts, (int64_t)s.rows * s.G <= z.own_rows);
  if (s.d == 64) join_shared<64>(P, z, stream);
  else if (s.d == 128) join_shared<128>(P, z, stream);
  else join_shared<256>(P, z, stream);
  return hipGetLastError();
}

}  // namespace ugbs
