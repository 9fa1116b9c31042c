// Attention of a batch whose requests list common first pages: these pages once for all rows of
// a group, the pages that are a request's own for its rows, and the join of both.
//
// A softmax over the keys of pages P u R is what the two sets give apart: with M, l and o the
// maximum, the sum and the weighted values of each, the result is
//   (2^(M_P - M) o_P + 2^(M_R - M) o_R) / (2^(M_P - M) l_P + 2^(M_R - M) l_R),  M = max(M_P, M_R),
// the join that parts along the pages need anyway.  What is won is bytes: a page of the prefix
// is read once for a tile of rows of a kv head, of all requests of the group, instead of once for each request: 64 rows
// (32 at d 256; 16 where the batch has no more).
//
// ugbs_cache_share finds, once a step, what the requests of a group have in common (their table
// rows are compared, so nothing but the table says what is shared) and lays the parts out,
// as ugbs_cache_attend does for itself; the launches of a layer only look their part up.
// What bounds it: a long prefix with many rows the matrix cores and the vector ALU (32 requests of 28/4 heads, d 128, behind
// 128K tokens: 81 to 88 us, 325 with every request alone, 44 at the rate of a large product); less of it the parts'
// starts and ends and the join (64 requests of 32/8 heads behind 8K tokens: 30 us, of which the join 5; 75 alone).
#include <algorithm>

#include "cache_rows.h"
#include "cache_tiles.h"

namespace ugbs {
namespace {

// More query rows of a request to a kv head than this fill their tiles (8 requests behind 8K tokens: of 80 rows 44 us alone,
// 36 together, of 128 rows 47.7 and 46.0).
constexpr int kMostRows = 128;

// (the join's grid: a workgroup for each row)
bool shares(const CacheShape& s) {
  return s.B > 1 && (int64_t)s.rows * s.G <= kMostRows && (int64_t)s.B * s.rows * s.H <= (1 << 20);
}

struct Sizes {
  int own_rows, prefix_rows;          // of a tile
  int64_t parts;                      // at most
  int64_t sum_rows;                   // rows of the parts' sums, at most
};

// (A group's tile of 17 to 32 live rows is one of tile_rows_many all the same; its parts are taken as what they are:
// shared_part.)
int prefix_tile_rows(int d, int64_t rows) { return rows <= 16 ? 16 : tile_rows_many(d); }

// More parts than tiles: by kTarget at most; a group has two requests at least.
Sizes sizes_of(const CacheShape& s) {
  const int64_t all = (int64_t)s.B * s.rows * s.G, groups = s.B / 2;
  Sizes z;
  z.own_rows = tile_rows(s);
  z.prefix_rows = prefix_tile_rows(s.d, all);
  z.parts = tiles_bound(s, z.own_rows) + s.Hkv * (all / z.prefix_rows + groups) + kTarget;
  z.sum_rows = 2 * s.Hkv * all + kTarget * std::max(z.own_rows, z.prefix_rows);
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
  share->own = reinterpret_cast<int4*>(take(2 * sizeof(int4) * s.B));
  share->prefix = reinterpret_cast<int4*>(take(2 * sizeof(int4) * s.B));
  share->part = reinterpret_cast<int4*>(take(2 * sizeof(int4) * z.parts));
  share->row = reinterpret_cast<int2*>(take(sizeof(int2) * s.B * s.rows * s.G));
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

// Sums over the workgroup of N numbers of each thread: in all, and before it.
template <int NW, int N>
__device__ __forceinline__ void sum_all(float (&x)[N], float (*s_wave)[NW]) {
#pragma unroll
  for (int y = 0; y < N; ++y) {
    x[y] = sum_wave(x[y]);
    if ((threadIdx.x & 63) == 0) s_wave[y][threadIdx.x >> 6] = x[y];
  }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < N; ++y) {
    x[y] = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v) x[y] += s_wave[y][v];
  }
}
template <int NW, int N>
__device__ __forceinline__ void sum_before(const int (&x)[N], int (&before)[N], int (&total)[N], int (*s_wave)[NW]) {
  const int w = threadIdx.x >> 6;
#pragma unroll
  for (int y = 0; y < N; ++y) {
    before[y] = scan_add(x[y]);
    if ((threadIdx.x & 63) == 63) s_wave[y][w] = before[y];
    before[y] -= x[y];
    total[y] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < N; ++y)
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      if (v < w) before[y] += s_wave[y][v];
      total[y] += s_wave[y][v];
    }
}

// What a part costs, in pages of a prefix part: its start and end; a page and the start of a part of own pages.
constexpr float kStart = 6.0f, kOwnPage = 0.75f, kOwnStart = 4.0f;
// Common pages are shared where that saves more pages a place than the rows' joins cost.  Without: 32 requests of up to 1000
// tokens behind 4 common pages (1.4 saved) 13.6 us, with 17.5; behind 16 (5.5) 17.6 and 18.7; 8 groups of 8 behind up to 64 each
// (23) 43.5 and 24.  Tiles that are the same for own pages save the bytes that several would read (kSameTile for 1): 8 requests of
// 64 rows behind 128 pages (4.0) 32.5 and 30.9.
constexpr float kSameTile = 1.25f, kLeastSaved = 7.0f, kLeastSame = 3.0f;
constexpr int kTimes = 8;                 // candidates for the longest part's time, each
constexpr float kLonger = 0.1f;           // so much longer than the one before

// The parts, PER requests a thread.  PER 1: every workgroup forms the requests' entries and sums for itself, in LDS, and
// writes its share (1000 requests, with the comparison: 15 us).  More: one workgroup, which finds its entries again in the plan
// (2000: 47, 4000: 80).  FIND: what share_compare_kernel does comes first here, for few requests of few pages.
template <int THREADS, int PER, bool FIND>
__global__ void __launch_bounds__(THREADS) share_plan_kernel(CacheAttendParams P, const int32_t* __restrict__ group, int own_rows,
                                                             int prefix_rows, int parts) {
  constexpr int NW = THREADS / 64, MOST = THREADS * PER;
  constexpr bool kMany = PER == 1;
  // new tokens, parts of a tile, rows of sums before, common pages; of the group the same; first entry in `row`, cached tokens
  __shared__ int4 s_own[kMany ? MOST : 1], s_pre[kMany ? MOST : 1];
  __shared__ int2 s_more[kMany ? MOST : 1];
  __shared__ int s_a[MOST], s_b[MOST], s_c[MOST];
  __shared__ float s_saved[1][NW], s_sum[5][NW], s_parts[kTimes][NW];
  __shared__ int s_scan[5][NW];
  const int tid = threadIdx.x, B = P.s.B, G = P.s.G, Hkv = P.s.Hkv, most = P.s.max_pages * kBlock;
  for (int b = tid; b < B; b += THREADS) {
    s_a[b] = INT32_MAX;
    s_b[b] = s_c[b] = 0;
  }
  int4 found[PER];
  Lengths own[PER], pre[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k;
    found[k] = make_int4(-1, 0, 0, 0);
    own[k] = pre[k] = Lengths{0, 0, 0, 0};
    if (b < B) {
      if constexpr (!FIND) found[k] = P.share.found[b];
      own[k].q = min(max(P.q_lens[b], 0), P.s.rows);
      own[k].kv = min(max(P.kv_lens[b], 0), most);
    }
  }
  if constexpr (FIND) {
    static_assert(PER == 1, "a request a thread");
    // (s_own: group or -1, new tokens, full pages, pages in common with the leader)
    const int mine = tid < B && own[0].q > 0 ? group[tid] : -1;
    s_own[tid] = make_int4(mine, own[0].q, own[0].kv / kBlock, INT32_MAX);
    __syncthreads();
    int members = 0, leader = -1;
    if (mine >= 0)
      for (int x = 0; x < B; ++x) {
        const int4 y = s_own[x];
        if (y.x != mine) continue;
        if (members++ == 0) leader = x;
        if (x < tid) found[0].z += y.y;
      }
    if (members > 1) {
      found[0].x = leader;
      s_own[tid].w = min(s_own[tid].z, s_own[leader].z);
    }
    s_more[tid].x = found[0].x;
    __syncthreads();
    const int width = P.s.max_pages;
    for (int i = tid; i < B * width; i += THREADS) {
      const int b = i / width, j = i - b * width, l = s_more[b].x;
      if (l >= 0 && l != b && j < s_own[b].w && P.table[(size_t)b * width + j] != P.table[(size_t)l * width + j]) atomicMin(&s_own[b].w, j);
    }
    __syncthreads();
    found[0].y = s_own[tid].w;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int l = found[k].x;
    if (l >= 0) {
      atomicMin(&s_a[l], found[k].y);                          // pages in common
      atomicMax(&s_b[l], found[k].z + own[k].q);               // new tokens
      atomicAdd(&s_c[l], 1);
    }
  }
  __syncthreads();
  const bool alike = own_rows == prefix_rows;
  const float cost = alike ? 1.0f : kOwnPage, start = alike ? kStart : kOwnStart;
  // (the last tile of a group may be one of few rows)
  auto prefix_work = [&](const Lengths& r) {
    const float few = prefix_rows > 32 && r.q * G - (r.tiles - 1) * prefix_rows <= 32 ? 1.0f - kOwnPage : 0.0f;
    return ((float)r.tiles - few) * (float)r.pages;
  };
  int together[PER];                                           // new tokens of the group
  float saved[1] = {0.f};
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k, l = found[k].x;
    together[k] = l >= 0 ? s_b[l] : 0;
    found[k].y = l >= 0 ? s_a[l] : 0;
    own[k].tiles = (own[k].q * G + own_rows - 1) / own_rows;
    saved[0] += (alike ? kSameTile : kOwnPage) * (float)(own[k].tiles * found[k].y);
    if (found[k].y > 0 && b == l) {
      pre[k].q = together[k];
      pre[k].tiles = (together[k] * G + prefix_rows - 1) / prefix_rows;
      pre[k].pages = found[k].y;
      saved[0] -= prefix_work(pre[k]);
    }
  }
  sum_all<NW>(saved, s_saved);
  if (saved[0] * (float)Hkv < (float)kTarget * (prefix_rows == 16 ? 0.0f : alike ? kLeastSame : kLeastSaved)) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      found[k].y = 0;
      pre[k] = Lengths{0, 0, 0, 0};
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) own[k].pages = max((own[k].kv + kBlock - 1) / kBlock - found[k].y, 0);
  // Pages a part, from the time that the longest may take: all parts together, spread evenly over the chip's
  // places, and longer until there is a place for each (where there are more tiles than places: as it is).
  float sums[5] = {0.f, 0.f, 0.f, 0.f, 0.f};                   // work and tiles, own and of prefixes; pages of all tiles
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    sums[0] = __builtin_fmaf((float)own[k].tiles, (float)own[k].pages, sums[0]);
    sums[1] += prefix_work(pre[k]);
    sums[2] += (float)own[k].tiles;
    sums[3] += (float)pre[k].tiles;
    sums[4] += (float)(own[k].tiles * own[k].pages + pre[k].tiles * pre[k].pages);
  }
  sum_all<NW>(sums, s_sum);
#pragma unroll
  for (int y = 0; y < 5; ++y) sums[y] *= (float)Hkv;
  const float least = (float)P.min_pages, each = 1.0f / kTarget;
  auto pages_of_time = [&](float time, int* o, int* p) {
    *o = *p = UGBS_MAX_BLOCKS;
    if (!P.splits) return;
    // (no more than kTarget parts above the tiles, own and of prefixes together)
    const float most = fmaxf(sums[4] * each, least), x = fmaxf((time - start) * __builtin_amdgcn_rcpf(cost), most), y = fmaxf(time - kStart, most);
    *o = x < (float)UGBS_MAX_BLOCKS ? (int)x + 1 : UGBS_MAX_BLOCKS;
    *p = y < (float)UGBS_MAX_BLOCKS ? (int)y + 1 : UGBS_MAX_BLOCKS;
  };
  // (x pages of a prefix in the longest part: time(x) = a + b / x, whose fixed point the geometric mean of both approaches
  // from one side)
  float x = fmaxf((cost * sums[0] + sums[1]) * each, 1.0f);
#pragma unroll
  for (int y = 0; y < 6; ++y) {
    const float n_o = fmaxf(sums[2], sums[0] * cost * __builtin_amdgcn_rcpf(fmaxf(x + kStart - start, 1.0f)));
    const float n_p = fmaxf(sums[3], sums[1] * __builtin_amdgcn_rcpf(x));
    const float t = (cost * sums[0] + sums[1] + start * n_o + kStart * n_p) * each - kStart;
    x = fmaxf(__builtin_amdgcn_sqrtf(x * fmaxf(t, 1.0f)), 1.0f);
  }
  const float time = x + kStart;
  float longer = 1.0f;
  if (sums[2] + sums[3] <= (float)kTarget) {
    // the first of kTimes candidates with a place for each part: `from`, `from` + step, ... (else the last one)
    auto fitting = [&](float from, float step) {
      float parts_at[kTimes];
#pragma unroll
      for (int y = 0; y < kTimes; ++y) {
        int o, p;
        pages_of_time(time * (from + step * y), &o, &p);
        const float io = __builtin_amdgcn_rcpf((float)o), ip = __builtin_amdgcn_rcpf((float)p);
        parts_at[y] = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k)
          parts_at[y] += own[k].tiles * fmaxf(ceilf(own[k].pages * io), 1.0f) + pre[k].tiles * fmaxf(ceilf(pre[k].pages * ip), 1.0f);
      }
      __syncthreads();
      sum_all<NW>(parts_at, s_parts);
      float found = from + step * (kTimes - 1);
#pragma unroll
      for (int y = kTimes - 2; y >= 0; --y)
        if (parts_at[y] * (float)Hkv <= (float)kTarget) found = from + step * y;
      return found;
    };
    longer = fitting(1.0f, kLonger);
    if (longer > 1.0f) longer = fitting(longer - kLonger, kLonger / (kTimes - 1));
  }
  int per_own, per_pre;
  pages_of_time(time * longer, &per_own, &per_pre);
  // parts and rows of sums of the requests and of the groups, and the groups' new tokens
  int n[5] = {0, 0, 0, 0, 0}, at[5], total[5];
  auto count = [&](int k, int (&x)[5]) {
    const int so = splits_of(own[k], per_own), sp = splits_of(pre[k], per_pre);
    x[0] = own[k].tiles * Hkv * so;
    x[1] = own[k].tiles > 0 && (so > 1 || found[k].y > 0) ? so * Hkv * own[k].q * G : 0;
    x[2] = pre[k].tiles * Hkv * sp;
    x[3] = sp * Hkv * pre[k].q * G;
    x[4] = pre[k].q;
  };
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    int x[5];
    count(k, x);
#pragma unroll
    for (int y = 0; y < 5; ++y) n[y] += x[y];
  }
  sum_before<NW>(n, at, total, s_scan);
  at[3] += total[1];                                           // behind the requests' own
  // (the barriers of the sums are behind the last reads of s_a and s_b)
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k, so = splits_of(own[k], per_own), sp = splits_of(pre[k], per_pre);
    int x[5];
    count(k, x);
    if (b < B) {
      s_a[b] = at[0];
      s_b[b] = at[2];
      const int4 o = make_int4(own[k].q, so, so > 1 || found[k].y > 0 ? at[1] : -1, found[k].y);
      const int4 p = make_int4(pre[k].q, sp, at[3], pre[k].pages);
      if (blockIdx.x == 0) P.share.own[2 * b] = o;
      if constexpr (kMany) {
        s_own[b] = o;
        s_pre[b] = p;
        s_more[b] = make_int2(at[4], own[k].kv);
      } else {
        P.share.prefix[2 * b] = p;
        P.share.prefix[2 * b + 1] = make_int4(at[4], own[k].kv, 0, 0);
      }
    }
#pragma unroll
    for (int y = 0; y < 5; ++y) at[y] += x[y];
  }
  __syncthreads();
  auto own_of = [&](int b) { return kMany ? s_own[kMany ? b : 0] : P.share.own[2 * b]; };
  auto prefix_of = [&](int b) { return kMany ? s_pre[kMany ? b : 0] : P.share.prefix[2 * b]; };
  auto more_of = [&](int b) {
    if constexpr (kMany) return s_more[b];
    const int4 x = P.share.prefix[2 * b + 1];
    return make_int2(x.x, x.y);
  };
  // what the join and the parts of prefixes look up
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k, l = found[k].x;
    if (b >= B || b % gridDim.x != blockIdx.x) continue;
    int4 y = make_int4(-1, 0, 0, 0);
    if (found[k].y > 0) {
      const int4 of = prefix_of(l);
      y = make_int4(of.z, of.y, found[k].z, together[k] * G);
      int2* const row = P.share.row + (size_t)(more_of(l).x + found[k].z) * G;
      for (int i = 0; i < own[k].q; ++i)
        for (int g = 0; g < G; ++g) row[i * G + g] = make_int2((b * P.s.H + g) * P.s.rows + i, own[k].kv - own[k].q + i);
    }
    P.share.own[2 * b + 1] = y;
  }
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
  // The list: the parts of prefixes, which are longer, first.  (Spread among the others, so that each CU has
  // one of each, 64 requests behind 8K tokens took 34.6 us for 32.9.)  Without gaps: kTarget parts are as many for each
  // XCD.  (With own parts from a multiple of 8 on, one XCD had 65 for its 64 places, and the last one waited for another's
  // end: 40 drafts of d 256 behind 5 prompts 69 us for 58.)
  for (int i = blockIdx.x * THREADS + tid; i < parts; i += gridDim.x * THREADS) {
    int4 x = make_int4(-1, 0, 0, 0), y = x;
    if (i < total[2] + total[0]) {
      const bool prefix = i < total[2];
      const int pos = prefix ? i : i - total[2];
      const int b = request_at(prefix ? s_b : s_a, pos);
      const int4 r = prefix ? prefix_of(b) : own_of(b);
      const int2 more = more_of(b);
      const int size = prefix ? prefix_rows : own_rows, rows = r.x * G, tiles = (rows + size - 1) / size;
      Part u;
      u.splits = r.y;
      if (prefix) locate<kGroups>(P, pos - s_b[b], tiles, 0, &u);
      else locate<kParts>(P, pos - s_a[b], tiles, 0, &u);
      const int row = r.z < 0 ? -1 : r.z + u.splits * (u.kvh * rows + u.tile * size) + u.split * min(size, rows - u.tile * size);
      int first = 0, pages = r.w;
      if (!prefix) {
        // pages that the tile's last row sees, behind the common ones
        const int end = more.y - r.x + (min((u.tile + 1) * size, rows) - 1) / G + 1;
        first = r.w;
        pages = max((max(end, 0) + kBlock - 1) / kBlock - first, 0);
      }
      x = make_int4(b, u.kvh + (prefix ? kOfPrefix : 0), u.tile, first + pages * u.split / u.splits);
      y = make_int4(first + pages * (u.split + 1) / u.splits, row, r.x, prefix ? more.x : more.y);
    }
    P.share.part[2 * i] = x;
    P.share.part[2 * i + 1] = y;
  }
}

// The parts of a layer: a workgroup looks its part up, and takes it as few or as many rows.
constexpr int kWaves = 4;
constexpr int tiles_rt(int d) { return d == 256 ? 2 : 4; }
constexpr int tiles_qr(int d) { return d == 64 ? 4 : 2; }
constexpr int tiles_waves(int d) { return d == 64 ? 3 : 2; }

template <int D, int DT, int ROWS>
struct Kind {                                     // tiles of ROWS rows
  static constexpr bool kMany = ROWS == tile_rows_many(D);
  using Few = RowsMemory<D, ROWS / 16, kWaves>;
  using Many = TilesMemory<D, DT, tiles_rt(D), tiles_qr(D), kWaves>;
  using Memory = std::conditional_t<kMany, Many, Few>;
  // ONCE: no other workgroup reads these bytes
  template <Mode MODE, bool ONCE>
  __device__ static __forceinline__ void part(const CacheAttendParams& P, const Part& u, int row, int p0, int p1, Memory& memory) {
    if constexpr (kMany) tiles_part<D, DT, tiles_rt(D), tiles_qr(D), kWaves, ONCE, MODE>(P, u, row, p0, p1, memory);
    else rows_part<D, DT, ROWS / 16, kWaves, MODE>(P, u, row, p0, p1, memory);
  }
};

template <int D, int DT, int PREFIX, int OWN>
__device__ __forceinline__ void shared_part(const CacheAttendParams& P) {
  __shared__ union Memory {
    typename Kind<D, DT, PREFIX>::Memory prefix;
    typename Kind<D, DT, OWN>::Memory own;
    typename Kind<D, DT, 16>::Memory few;
    typename Kind<D, DT, PREFIX < 32 ? 16 : 32>::Memory some;
    std::conditional_t<(PREFIX > 32), TilesMemory<D, DT, 2, 2, kWaves>, int> half;
  } memory;
  const int4 x = P.share.part[2 * blockIdx.x], y = P.share.part[2 * blockIdx.x + 1];
  auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  Part u;
  u.b = same(x.x);
  if (u.b < 0) return;
  u.kvh = same(x.y);
  u.tile = same(x.z);
  u.q = same(y.z);
  const int p0 = same(x.w), p1 = same(y.x), row = same(y.y), last = same(y.w);
  if (u.kvh >= kOfPrefix) {
    u.kvh -= kOfPrefix;
    u.slot = last;
    u.kv = p1 * kBlock;
    // Few rows cost less as what they are.  A group's only tile reads bytes that no other one does: straight into
    // registers (4 requests of 7 rows behind 128K: 35 us, 38.5 as a half tile through LDS, 40 as a tile of 64); the last one of
    // several shares them (32 requests of 7 rows: 90, 82 and 86 us).
    const int live = u.q * P.s.G - u.tile * PREFIX;
    if constexpr (PREFIX > 16)
      if (live <= 16 && u.tile == 0) return Kind<D, DT, 16>::template part<kPrefix, true>(P, u, row, p0, p1, memory.few);
    if constexpr (PREFIX > 32)
      if (live <= 32) {
        if (u.tile == 0) return Kind<D, DT, 32>::template part<kPrefix, true>(P, u, row, p0, p1, memory.some);
        u.tile *= 2;
        return tiles_part<D, DT, 2, 2, kWaves, false, kPrefix>(P, u, row, p0, p1, memory.half);
      }
    // (8 requests of 7 rows behind 128K: 39 us for 44 with the bytes kept in the caches; of several tiles none passes them: 32
    // requests of 8 rows at d 256 behind 30K 32.1 us for 32.8 with the first one past them, 40 of 32 in 5 groups 43.3 for 46.2, in
    // int8 57 either way, 64 of 4 at d 128 behind 8K 29.9 for 30.1)
    if (u.q * P.s.G <= PREFIX) Kind<D, DT, PREFIX>::template part<kPrefix, true>(P, u, row, p0, p1, memory.prefix);
    else Kind<D, DT, PREFIX>::template part<kPrefix, false>(P, u, row, p0, p1, memory.prefix);
  } else {
    u.kv = last;
    // (tiles of many rows stay in the caches: a request may have several, and one alone is no slower, 27.2 us for 28.5 with
    // 8 requests of 64 rows and up to 8000 tokens)
    Kind<D, DT, OWN>::template part<kOwn, false>(P, u, row, p0, p1, memory.own);
  }
}

template <int D, int DT, int OWN>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(tiles_waves(D), tiles_waves(D))))
shared_tiles_kernel(CacheAttendParams P) {
  shared_part<D, DT, tile_rows_many(D), OWN>(P);
}
template <int D, int DT>
__global__ void __launch_bounds__(64 * kWaves) shared_rows_kernel(CacheAttendParams P) {
  shared_part<D, DT, 16, 16>(P);
}

template <int D, int DT>
void shared_parts(const CacheAttendParams& P, const Sizes& z, hipStream_t stream) {
  const unsigned n = (unsigned)z.parts;
  if (z.prefix_rows == 16) shared_rows_kernel<D, DT><<<n, 64 * kWaves, 0, stream>>>(P);
  else if (z.own_rows == 16) shared_tiles_kernel<D, DT, 16><<<n, 64 * kWaves, 0, stream>>>(P);
  else if (z.own_rows == 32) shared_tiles_kernel<D, DT, 32><<<n, 64 * kWaves, 0, stream>>>(P);
  else if constexpr (D != 256) shared_tiles_kernel<D, DT, 64><<<n, 64 * kWaves, 0, stream>>>(P);
}

// Joins the parts of the rows of a request, those of the prefix first: NT threads to a row, D / 4 to a
// part of it, eight parts of a thread on their way at once.
template <int D, int NT>
__global__ void __launch_bounds__(256) share_join_kernel(CacheAttendParams P, int own_rows, int prefix_rows) {
  constexpr int CG = D / 4, GR = NT / CG, ROWS = 256 / NT, W = NT / 64, kAhead = 8;
  constexpr int kMost = kTarget + 2;        // parts of a row
  __shared__ float s_weight[ROWS][kMost];
  __shared__ float2 s_ml[4];
  __shared__ f32x4 s_o[W > 1 ? GR : 1][CG];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, G = P.s.G;
  const int b = blockIdx.x / P.s.Hkv, kvh = blockIdx.x % P.s.Hkv, mine = tid / NT, t = tid % NT;
  const int r = blockIdx.y * ROWS + mine;
  const int4 x = P.share.own[2 * b], y = P.share.own[2 * b + 1];
  // (a row's threads leave together: no barrier where there is a wave or less to a row)
  if (x.z < 0 || r >= x.x * G) return;
  const int all = x.x * G, tile = r / own_rows;
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

// The fewer rows, the more parts of each: 112 rows of some 100 parts take 8 us with a workgroup to a row, 24 with a
// wave; 2048 rows of 9 parts 6.3 and 4.5.
template <int D>
void join_shared(const CacheAttendParams& P, const Sizes& z, hipStream_t stream) {
  const int rows = P.s.rows * P.s.G, units = P.s.B * P.s.Hkv;
  if (units * rows < 1024) share_join_kernel<D, 256><<<dim3(units, rows), 256, 0, stream>>>(P, z.own_rows, z.prefix_rows);
  else share_join_kernel<D, 64><<<dim3(units, (rows + 3) / 4), 256, 0, stream>>>(P, z.own_rows, z.prefix_rows);
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
  const bool few = s.B <= 64 && s.B * s.max_pages <= 4096;
  if (!few) share_compare_kernel<<<(unsigned)s.B, 256, 0, stream>>>(P, group);
  auto blocks = [&](int threads) { return (unsigned)std::min<int64_t>((z.parts + threads - 1) / threads, 16); };
  const int parts = (int)z.parts;
  if (few) share_plan_kernel<256, 1, true><<<blocks(256), 256, 0, stream>>>(P, group, z.own_rows, z.prefix_rows, parts);
  else if (s.B <= 256) share_plan_kernel<256, 1, false><<<blocks(256), 256, 0, stream>>>(P, group, z.own_rows, z.prefix_rows, parts);
  else if (s.B <= 1024) share_plan_kernel<1024, 1, false><<<blocks(1024), 1024, 0, stream>>>(P, group, z.own_rows, z.prefix_rows, parts);
  else share_plan_kernel<1024, UGBS_MAX_REQUESTS / 1024, false><<<1, 1024, 0, stream>>>(P, group, z.own_rows, z.prefix_rows, parts);
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
  const bool f8 = s.dtype == UGBS_E4M3;
  if (s.d == 64) (f8 ? shared_parts<64, UGBS_E4M3> : shared_parts<64, UGBS_INT8>)(P, z, stream);
  else if (s.d == 128) (f8 ? shared_parts<128, UGBS_E4M3> : shared_parts<128, UGBS_INT8>)(P, z, stream);
  else (f8 ? shared_parts<256, UGBS_E4M3> : shared_parts<256, UGBS_INT8>)(P, z, stream);
  if (s.d == 64) join_shared<64>(P, z, stream);
  else if (s.d == 128) join_shared<128>(P, z, stream);
  else join_shared<256>(P, z, stream);
  return hipGetLastError();
}

}  // namespace ugbs
