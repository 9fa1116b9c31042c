// What the kernels of the attention over the cache share: the parts of a call, the
// pages of a part, the join.
#pragma once
#include "cache_internal.h"

namespace ugbs {

// Parts a call aims at, at most, and the pages of a part, at least: 64 KiB at d 64 and 128,
// 128 KiB at d 256 (one request of 4000 tokens at d 128: 11.3 us with 8 pages, 10.1 with 4; of 8000 at
// d 256: 11.7 with 4, 12.4 with 2).
constexpr int kTarget = 512;
constexpr int min_pages(int d) { return d == 64 ? 8 : 4; }
// Parts of split tiles are at most twice W / X, X > W / kTarget, and a split tile has at least two.
constexpr int kSlots = 2 * kTarget;
// A tile with more parts than kLongParts is long: joined by a workgroup for each row
// (of 64 rows: for every fourth at least), also among many tiles.
constexpr int kLongParts = 32, kLongTiles = kSlots / (kLongParts + 1);

// Where the parts lie, of batches of more than kWaveBatch requests: formed once by
// cache_schedule_kernel, in the workspace.  Up to kWaveBatch every wave forms it for itself
// (4 lengths a lane), which is quicker than a launch.
constexpr int kWaveBatch = 256;
struct Schedule {
  int4* request;      // [B]: parts before, parts of a tile, slots before, split tiles before
  int32_t* part;      // [tiles + kTarget]: the request, -1 behind the last part
  int32_t* join;      // [kTarget]: the same for the split tiles
  int2* long_tile;    // [kLongTiles]: request (-1 behind the last), which of its tiles
};

// Where the parts lie of a batch whose requests list common first pages: formed once a step by
// ugbs_cache_share.  A group of such requests has a leader, its first one.  The rows of a part's sums
// lie in the workspace one behind another: part `split` of tile t of kv head h, R rows in all, begins at row
//   before + splits (h R + t ROWS) + split min(ROWS, R - t ROWS).
struct Share {
  int4* own;          // [B][2]: (new tokens, parts of a tile, rows before or -1: written to O, common pages),
                      //   (rows before of its group's prefix or -1, parts of a tile there, first new token in the group, group's R)
  int4* prefix;       // [B][2], of leaders: (new tokens, parts of a tile, rows before, pages), (first entry in `row`; its own cached tokens, -, -)
  int4* part;         // [parts][2]: (request or leader, -1: none; kv head, of a prefix + kOfPrefix; tile; first page),
                      //   (behind its last page; row of its sums or -1; new tokens; cached tokens or, of a prefix, first entry in `row`)
  int2* row;          // [B rows G]: rows of the groups: where its query of the first kv head lies (a row of Q), the last key it sees
  int4* found;        // [B]: leader (-1: alone), pages in common with it, new tokens of the group's requests before
};
constexpr int kOfPrefix = 1 << 24;

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
  Schedule schedule;  // of more than kWaveBatch requests
  int min_pages;
  Share share;        // of common first pages
};

// What a launch of the parts takes: whole requests; the pages that are a request's own, those that groups
// have in common (ugbs_cache_attend_shared).
enum Mode { kWhole, kOwn, kPrefix };

// Tiles of 64 (d 256: 32) rows, where rows are many (cache_tiles.hip).
hipError_t launch_cache_tiles(const CacheAttendParams& P, hipStream_t stream);
constexpr int tile_rows_many(int d) { return d == 256 ? 32 : 64; }

namespace {

constexpr float kNoMax = -3.402823466e38f;     // a row's maximum before its first key

__device__ __forceinline__ float sum_groups(float x) {    // over lanes l, l ^ 16, l ^ 32, l ^ 48 (those that hold a row)
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ float sum_wave(float x) {      // over all lanes
  auto add = [&](int y) { x += __uint_as_float((unsigned)y); };
  add(dpp<0xb1, 0xf>((int)__float_as_uint(x)));           // lane ^ 1
  add(dpp<0x4e, 0xf>((int)__float_as_uint(x)));           // lane ^ 2
  add(dpp<0x141, 0xf>((int)__float_as_uint(x)));          // 7 - lane, within 8
  add(dpp<0x140, 0xf>((int)__float_as_uint(x)));          // 15 - lane, within 16
  return sum_groups(x);
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

// Pages per part, from the sums over the requests of tiles times pages, of tiles and of
// wide tiles (fp32, added in the same order wherever they are formed; + 1 covers the
// rounding, X being at most 4096).  Each tile ends with a part that is not full, half a part on
// average, and kTarget parts are two a CU: half the tiles are taken off, so that few CUs get a
// third (16 requests of up to 8000, 128 tiles: 36.0 -> 32.5 us; 32 ragged ones, 256 tiles: 57.1 ->
// 54.6).  At 64 rows two are all that a CU holds at once, and a third is a second round: there
// three quarters of the tiles are taken off (56 tiles: as 560 parts 264 us, as 504 193).  Tiles
// of a few pages among long ones end no part that matters and are not counted (one request
// of 100K among 3 of 100, 64 rows of 64/16 heads, d 64: 220 -> 156 us).
__device__ __forceinline__ int pages_per_part(const CacheAttendParams& P, int rows, float work, float tiles, float wide) {
  if (!P.splits) return UGBS_MAX_BLOCKS;
  const float off = (rows <= 32 ? 0.5f : 0.75f) * wide * (float)P.s.Hkv;
  const float aim = fmaxf((float)kTarget - off, 0.5f * kTarget);
  const float x = work * (float)P.s.Hkv / aim;
  // (256 tiles fill the chip: 512 tokens attending to themselves 26 us split, 20 whole)
  const int least = tiles * (float)P.s.Hkv < 0.5f * kTarget ? P.min_pages : 2 * P.min_pages;
  return x < (float)UGBS_MAX_BLOCKS ? max((int)x + 1, least) : UGBS_MAX_BLOCKS;
}
// Wide: of at least a quarter of work / kTarget pages.
__device__ __forceinline__ bool is_wide(const CacheAttendParams& P, const Lengths& r, float work) {
  return (float)r.pages * (4 * kTarget) > work * (float)P.s.Hkv;
}
__device__ __forceinline__ int splits_of(const Lengths& r, int per) { return r.pages > per ? (r.pages + per - 1) / per : 1; }

// Part number pos of the call (kJoinTiles: tile number pos among the split ones,
// kLongTilesOnly: among the long ones).
// The parts of a request follow each other.  kParts: kv head, tile, part.  kGroups:
// tiles that read the same pages (kv head, part) on one XCD, one after another, so
// that its L2 serves all but the first: workgroup j runs on XCD j mod 8, so groups
// are dealt out 8 at a time, those that are left over in turn (4 of them keep to two XCDs each; in a
// row they run on all 8: drafts of d 256 behind 5 prompts, 14 draws, 58.7 us, in turn 57.5; 25 kinds of pieces of prompts in
// a row 1.4% less to 3.6% more, 42 of 1014 tokens of 28/4 heads 320 us, in turn 316).  Uniform over the wave.
enum Order { kParts, kGroups, kJoinTiles, kLongTilesOnly };
template <Order ORDER>
__device__ __forceinline__ void locate(const CacheAttendParams& P, int at, int tiles, int slots_before, Part* out) {
  out->split = 0;
  if (ORDER == kGroups) {
    const int groups = P.s.Hkv * out->splits, dealt = groups / 8 * 8;
    int group;
    if (at < dealt * tiles) {
      group = at / 8 / tiles * 8 + at % 8;
      out->tile = at / 8 % tiles;
    } else {
      const int rest = at - dealt * tiles, left = groups - dealt;
      group = dealt + rest % left;
      out->tile = rest / left;
    }
    out->tile = tiles - 1 - out->tile;      // later rows see more: first
    out->split = group % out->splits;
    out->kvh = group / out->splits;
  } else {
    if (ORDER == kParts) {
      out->split = at % out->splits;
      at /= out->splits;
    }
    out->tile = at % tiles;
    out->kvh = at / tiles;
  }
  out->slot = slots_before + (out->kvh * tiles + out->tile) * out->splits;
}

template <int ROWS, Order ORDER>
__device__ bool find_part(const CacheAttendParams& P, int pos, Part* out) {
  const int lane = threadIdx.x & 63, B = P.s.B, Hkv = P.s.Hkv;
  if (B > kWaveBatch) {
    if ((ORDER == kJoinTiles && pos >= kTarget) || (ORDER == kLongTilesOnly && pos >= kLongTiles)) return false;
    const int b = __builtin_amdgcn_readfirstlane(ORDER == kLongTilesOnly ? P.schedule.long_tile[pos].x
                                                                         : (ORDER == kJoinTiles ? P.schedule.join : P.schedule.part)[pos]);
    if (b < 0) return false;
    const int4 x = P.schedule.request[b];
    const Lengths r = lengths_of<ROWS>(P, b);
    out->b = b;
    out->q = r.q;
    out->kv = r.kv;
    out->splits = x.y;
    locate<ORDER>(P, ORDER == kLongTilesOnly ? P.schedule.long_tile[pos].y : pos - (ORDER == kJoinTiles ? x.w : x.x), r.tiles, x.z, out);
    return true;
  }
  constexpr int NC = kWaveBatch / 64;
  Lengths r[NC];
  float work = 0.f, tiles = 0.f;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    r[k] = Lengths{0, 0, 0, 0};
    if (64 * k + lane < B) r[k] = lengths_of<ROWS>(P, 64 * k + lane);
  }
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    work = __builtin_fmaf((float)r[k].tiles, (float)r[k].pages, work);
    tiles += (float)r[k].tiles;
  }
  work = sum_wave(work);
  float wide = 0.f;
#pragma unroll
  for (int k = 0; k < NC; ++k)
    if (is_wide(P, r[k], work)) wide += (float)r[k].tiles;
  const int per = __builtin_amdgcn_readfirstlane(pages_per_part(P, ROWS, work, sum_wave(tiles), sum_wave(wide)));
  int before = 0, slots = 0;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    if (64 * k >= B) return false;
    const int splits = splits_of(r[k], per), units = r[k].tiles * Hkv;
    const int used = splits > 1 ? units * splits : 0;
    const int mine = ORDER == kJoinTiles       ? (splits > 1 ? units : 0)
                     : ORDER == kLongTilesOnly ? (splits > kLongParts ? units : 0)
                                               : units * splits;
    const int upto = before + scan_add(mine), slots_upto = slots + scan_add(used);
    const unsigned long long found = __ballot(pos >= upto - mine && pos < upto);
    if (found) {
      const int l = __builtin_ctzll(found);
      out->b = 64 * k + l;
      out->q = __builtin_amdgcn_readlane(r[k].q, l);
      out->kv = __builtin_amdgcn_readlane(r[k].kv, l);
      out->splits = __builtin_amdgcn_readlane(splits, l);
      locate<ORDER>(P, pos - __builtin_amdgcn_readlane(upto - mine, l), __builtin_amdgcn_readlane(r[k].tiles, l),
                    __builtin_amdgcn_readlane(slots_upto - used, l), out);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
    slots = __builtin_amdgcn_readlane(slots_upto, 63);
  }
  return false;
}

// The schedule of a large batch.  Every workgroup forms the sums over all requests (4 a
// thread) and then finds the request of its share of the parts by bisection.
constexpr int kScheduleThreads = 1024;
template <int ROWS>
__global__ void __launch_bounds__(kScheduleThreads) cache_schedule_kernel(CacheAttendParams P, int entries) {
  constexpr int PER = UGBS_MAX_REQUESTS / kScheduleThreads, NW = kScheduleThreads / 64;
  __shared__ int s_parts[UGBS_MAX_REQUESTS], s_joins[UGBS_MAX_REQUESTS];
  __shared__ int s_wave[4][NW];
  __shared__ float2 s_work[NW];
  __shared__ float s_wide[NW];
  const int tid = threadIdx.x, w = tid >> 6, B = P.s.B, Hkv = P.s.Hkv;
  Lengths r[PER];
  float work = 0.f, tiles = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k;
    r[k] = Lengths{0, 0, 0, 0};
    if (b < B) r[k] = lengths_of<ROWS>(P, b);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    work = __builtin_fmaf((float)r[k].tiles, (float)r[k].pages, work);
    tiles += (float)r[k].tiles;
  }
  work = sum_wave(work);
  tiles = sum_wave(tiles);
  if ((tid & 63) == 0) s_work[w] = make_float2(work, tiles);
  __syncthreads();
  work = tiles = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    work += s_work[v].x;
    tiles += s_work[v].y;
  }
  float wide = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (is_wide(P, r[k], work)) wide += (float)r[k].tiles;
  wide = sum_wave(wide);
  if ((tid & 63) == 0) s_wide[w] = wide;
  __syncthreads();
  wide = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) wide += s_wide[v];
  const int per = pages_per_part(P, ROWS, work, tiles, wide);
  int n[4] = {0, 0, 0, 0};                  // parts, slots, split tiles, long tiles
  int splits[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    splits[k] = splits_of(r[k], per);
    const int units = r[k].tiles * Hkv;
    n[0] += units * splits[k];
    if (splits[k] > 1) {
      n[1] += units * splits[k];
      n[2] += units;
    }
    if (splits[k] > kLongParts) n[3] += units;
  }
  int at[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int in = scan_add(n[x]);
    at[x] = in - n[x];
    if ((tid & 63) == 63) s_wave[x][w] = in;
  }
  __syncthreads();
  int total[4] = {0, 0, 0, 0};
#pragma unroll
  for (int v = 0; v < NW; ++v)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (v < w) at[x] += s_wave[x][v];
      total[x] += s_wave[x][v];
    }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int b = PER * tid + k;
    if (b < B) {
      s_parts[b] = at[0];
      s_joins[b] = at[2];
      if (blockIdx.x == 0) P.schedule.request[b] = make_int4(at[0], splits[k], at[1], at[2]);
      const int units = r[k].tiles * Hkv;
      at[0] += units * splits[k];
      if (splits[k] > 1) {
        at[1] += units * splits[k];
        at[2] += units;
      }
      if (blockIdx.x == 0 && splits[k] > kLongParts)
        for (int i = 0; i < units; ++i) P.schedule.long_tile[at[3]++] = make_int2(b, i);
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
  for (int i = blockIdx.x * kScheduleThreads + tid; i < entries; i += gridDim.x * kScheduleThreads)
    P.schedule.part[i] = i < total[0] ? request_at(s_parts, i) : -1;
  if (blockIdx.x == 0 && tid >= total[3] && tid < kLongTiles) P.schedule.long_tile[tid] = make_int2(-1, 0);
  if (blockIdx.x == 0 && tid < kTarget) P.schedule.join[tid] = tid < total[2] ? request_at(s_joins, tid) : -1;
}

// Row r of a part of a prefix: its row of Q, the last key it sees; (0, -1): there is none.
__device__ __forceinline__ int2 row_of(const CacheAttendParams& P, const Part& u, int r) {
  if (r >= u.q * P.s.G) return make_int2(0, -1);
  const int2 at = P.share.row[(size_t)u.slot * P.s.G + r];
  return make_int2(at.x + u.kvh * P.s.G * P.s.rows, at.y);
}

// Pages that the rows of a tile see (the last row sees most).
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

// The pages of a part that one wave visits (p, p + step, ...), 64 at a time, one a
// lane: its number and scales.  Entries that are no page are passed over.
struct Pages {
  const int32_t* row;
  const float* scales;                      // of this kv head
  int n_pages, stride, step, end;
  int first;                                // page of lane 0
  int id;
  float2 scale;
  unsigned long long left;                  // lanes whose page is still to visit

  __device__ __forceinline__ void load() {
    const int lane = threadIdx.x & 63;
    for (;;) {
      const int p = first + step * lane;
      id = p < end ? row[p] : -1;
      left = __ballot(id >= 0 && id < n_pages);
      if (left || first + 64 * step >= end) break;
      first += 64 * step;
    }
    scale = make_float2(0.f, 0.f);
    if (left >> lane & 1) scale = *reinterpret_cast<const float2*>(scales + (size_t)id * stride);
  }
  __device__ __forceinline__ void advance() {      // the next 64, if there are any
    if (first + 64 * step < end) {
      first += 64 * step;
      load();
    }
  }
  __device__ __forceinline__ int pop() {
    const int l = __builtin_ctzll(left);
    left &= left - 1;
    return l;
  }
  // the next lane to visit, -1: none; the lanes may then be others
  __device__ __forceinline__ int next() {
    if (!left) advance();
    return left ? pop() : -1;
  }
  __device__ __forceinline__ int page(int l) const { return __builtin_amdgcn_readlane(id, l); }
  __device__ __forceinline__ int at(int l) const { return first + step * l; }
  __device__ __forceinline__ float key_scale(int l) const {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale.x), l));
  }
  __device__ __forceinline__ float value_scale(int l) const {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale.y), l));
  }
};

__device__ __forceinline__ Pages pages_of(const CacheAttendParams& P, const Part& u, int p0, int p1, int first, int step) {
  Pages x;
  x.row = P.table + (size_t)u.b * P.s.max_pages;
  x.scales = P.scales + 2 * u.kvh;
  x.n_pages = P.s.n_pages;
  x.stride = 2 * P.s.Hkv;
  x.step = step;
  x.end = p1;
  x.first = p0 + first;
  x.load();
  return x;
}

// Lane masks of the values' bytes of a half page from position key0 on: those
// behind the last token may be anything and become 0 (a probability of 0 does not
// make them harmless).
__device__ __forceinline__ uint2 live_bytes(int kv, int key0) {
  const int g = (threadIdx.x & 63) >> 4;
  uint32_t keep[2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const int left = kv - (key0 + 16 * kt + 4 * g);
    keep[kt] = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
  }
  return make_uint2(keep[0], keep[1]);
}

__device__ __forceinline__ void store_row(const CacheAttendParams& P, const Part& u, int D, int at_row, int c, const f32x4& o, float inv) {
  const int i = at_row / P.s.G, h = u.kvh * P.s.G + at_row % P.s.G;
  *reinterpret_cast<uint2*>(P.O + (((size_t)u.b * P.s.H + h) * P.s.rows + i) * D + c) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

// The waves' sums of a part: O, or (row >= 0) rows `row` .. of the workspace.  seen: a key of the row has been
// looked at.  Each wave brings its own to the rows' maxima first (and, where the part is
// the whole, divides by the sums), so what is left are plain sums, 16 rows at a time, of
// values that lie in LDS as the lanes hold them.  s_o: NW D 16 floats, 16-byte aligned, may be
// what the waves still use on entry; s_ml: [NW][16 RT], may not.
template <int D, int RT, int NW>
__device__ __forceinline__ void finish_part(const CacheAttendParams& P, const Part& u, int64_t row, float* s_o, float2* s_ml,
                                            f32x4 (&acc)[RT][D / 16], const float (&m_run)[RT], const float (&l_run)[RT],
                                            const bool (&seen)[RT]) {
  constexpr int ROWS = 16 * RT, DT = D / 16;
  const CacheShape& s = P.s;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c16 = lane & 15;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = sum_groups(l_run[rt]);
    if (g == 0) s_ml[w * ROWS + 16 * rt + c16] = make_float2(seen[rt] ? m_run[rt] : -__builtin_huge_valf(), l);
  }
  __syncthreads();
  f32x4* const so = reinterpret_cast<f32x4*>(s_o);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int rr = 16 * rt + c16;
    float M = -__builtin_huge_valf(), l = 0.f, mine = 0.f;
    float2 ml[NW];
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      ml[v] = s_ml[v * ROWS + rr];
      M = fmaxf(M, ml[v].x);
    }
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float a = ml[v].x == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(ml[v].x - M);
      l += a * ml[v].y;
      if (v == w) mine = a;
    }
    if (row < 0) mine *= reciprocal(M, l);
    else if (w == 0 && g == 0 && u.tile * ROWS + rr < u.q * s.G) P.part_ml[row + rr] = make_float2(M, l);
    if (rt > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f32x4 x = acc[rt][dt];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= mine;
      so[(w * DT + dt) * 64 + lane] = x;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < DT / NW; ++k) {
      const int dt = k * NW + w, at_row = u.tile * ROWS + rr, c = 16 * dt + 4 * g;
      if (at_row < u.q * s.G) {
        f32x4 o = so[dt * 64 + lane];
#pragma unroll
        for (int v = 1; v < NW; ++v) o += so[(v * DT + dt) * 64 + lane];
        if (row < 0) store_row(P, u, D, at_row, c, o, 1.0f);
        else *reinterpret_cast<f32x4*>(P.part_o + (row + rr) * D + c) = o;
      }
    }
  }
}

// Joins the parts of row rr of a split tile: the work of a workgroup, D / 4 threads to a
// part, the parts round its threads; the first kAhead parts of a thread are on their way before
// the weights are known.  May be called again for another row without a barrier between.
template <int D, int ROWS>
__device__ __forceinline__ void join_row(const CacheAttendParams& P, const Part& u, int rr) {
  constexpr int CG = D / 4, GR = 256 / CG, kAhead = 16;
  __shared__ float2 s_part[kSlots / 2];     // maximum, then weight; sum
  __shared__ float2 s_ml[4];
  __shared__ f32x4 s_o[GR][CG];
  const int tid = threadIdx.x, w = tid >> 6, at_row = u.tile * ROWS + rr;
  if (at_row >= u.q * P.s.G) return;
  const int gr = tid / CG, c = tid % CG, splits = __builtin_amdgcn_readfirstlane(u.splits);
  const float2* const ml = P.part_ml + (size_t)u.slot * ROWS + rr;
  const f32x4* const po = reinterpret_cast<const f32x4*>(P.part_o + ((size_t)u.slot * ROWS + rr) * D) + c;
  float M = -__builtin_huge_valf();
  for (int v = tid; v < splits; v += 256) {
    s_part[v] = ml[(size_t)v * ROWS];
    M = fmaxf(M, s_part[v].x);
  }
  f32x4 ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (k * GR < splits) ahead[k] = po[(size_t)min(gr + k * GR, splits - 1) * (ROWS * CG)];
#pragma unroll
  for (int o = 1; o < 64; o *= 2) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) s_ml[w].x = M;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < 4; ++v) M = fmaxf(M, s_ml[v].x);
  float l = 0.f;
  for (int v = tid; v < splits; v += 256) {
    const float2 x = s_part[v];
    // a part that saw none of the row's keys weighs nothing
    const float a = x.x == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(x.x - M);
    s_part[v].x = a;
    if (a != 0.f) l += a * x.y;
  }
  l = sum_wave(l);
  if ((tid & 63) == 0) s_ml[w].y = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int v = 0; v < 4; ++v) l += s_ml[v].y;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](int v, const f32x4& x) {
    const float a = s_part[v].x;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += a * x[e];
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (gr + k * GR < splits) add(gr + k * GR, ahead[k]);
#pragma unroll 4
  for (int v = gr + kAhead * GR; v < splits; v += GR) add(v, po[(size_t)v * (ROWS * CG)]);
  s_o[gr][c] = o;
  __syncthreads();
  if (gr == 0) {
#pragma unroll
    for (int v = 1; v < GR; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += s_o[v][c][e];
    store_row(P, u, D, at_row, 4 * c, o, reciprocal(M, l));
  }
}

// Few tiles, which can have many parts: a workgroup for each row that there could be.
template <int D, int ROWS>
__global__ void __launch_bounds__(256) cache_join_kernel(CacheAttendParams P) {
  Part u;
  if (find_part<ROWS, kJoinTiles>(P, blockIdx.x, &u)) join_row<D, ROWS>(P, u, blockIdx.y);
}

// Many tiles, most of which have few parts: 1024 / D rows of a tile a workgroup, D / 4
// threads to a row, which take its parts eight at a time; nothing is shared.  (256 tiles
// of 64 rows in two parts each: 25 us with the kernel above, 5 with this one.)  LONG:
// behind the workgroups of `tiles` tiles come those of the long ones, `each` times as many
// a tile (one request of 200K tokens among 63 of 100, 8/1 heads: 95 us without them, 21 with; they
// cost up to 3 us where no tile is long).
template <int D, int ROWS, bool LONG>
__global__ void __launch_bounds__(256) cache_join_rows_kernel(CacheAttendParams P, int tiles, int each) {
  constexpr int CG = D / 4, kAhead = 8;
  // one wave looks the tile up: where no tile is split, that is all that 4096 workgroups do
  __shared__ Part s_u;
  __shared__ int s_found;
  const int past = LONG ? (int)blockIdx.x - tiles : -1;
  if (threadIdx.x < 64) {
    Part x;
    bool found;
    if constexpr (LONG) found = past < 0 ? find_part<ROWS, kJoinTiles>(P, blockIdx.x, &x) : find_part<ROWS, kLongTilesOnly>(P, past / each, &x);
    else found = find_part<ROWS, kJoinTiles>(P, blockIdx.x, &x);
    if (threadIdx.x == 0) {
      s_found = found;
      if (found) s_u = x;
    }
  }
  __syncthreads();
  if (!s_found) return;
  const Part u = s_u;
  if constexpr (LONG)
    if (past >= 0) {
      for (int rr = past % each * gridDim.y + blockIdx.y; rr < ROWS; rr += each * gridDim.y) join_row<D, ROWS>(P, u, rr);
      return;
    }
  const int splits = __builtin_amdgcn_readfirstlane(u.splits);
  if (LONG && splits > kLongParts) return;
  const int tid = threadIdx.x, rr = blockIdx.y * (256 / CG) + tid / CG, c = tid % CG, at_row = u.tile * ROWS + rr;
  if (rr >= ROWS || at_row >= u.q * P.s.G) return;
  const float2* const ml = P.part_ml + (size_t)u.slot * ROWS + rr;
  const f32x4* const po = reinterpret_cast<const f32x4*>(P.part_o + ((size_t)u.slot * ROWS + rr) * D) + c;
  float M = -__builtin_huge_valf(), l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int v = 0; v < splits; v += kAhead) {
    float2 x[kAhead];
    f32x4 y[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      x[k] = make_float2(-__builtin_huge_valf(), 0.f);
      if (v + k < splits) {
        x[k] = ml[(size_t)(v + k) * ROWS];
        y[k] = po[(size_t)(v + k) * (ROWS * CG)];
      }
    }
    float m = M;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) m = fmaxf(m, x[k].x);
    const float alpha = M == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(M - m);
    M = m;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= alpha;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v + k < splits && x[k].x != -__builtin_huge_valf()) {   // else the part saw none of the row's keys
        const float a = __builtin_amdgcn_exp2f(x[k].x - m);
        l += a * x[k].y;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += a * y[k][e];
      }
  }
  store_row(P, u, D, at_row, 4 * c, o, reciprocal(M, l));
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

inline bool may_split(const CacheShape& s) { return s.max_pages > min_pages(s.d); }

// Rows of a tile: as many as the call can have.
inline int tile_rows(int d, int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : tile_rows_many(d); }
inline int tile_rows(const CacheShape& s) { return tile_rows(s.d, (int64_t)s.rows * s.G); }

inline int64_t tiles_bound(const CacheShape& s, int rows_of_a_tile) {
  return (int64_t)s.B * s.Hkv * (((int64_t)s.rows * s.G + rows_of_a_tile - 1) / rows_of_a_tile);
}

// Entries of a schedule's list of parts.
inline int64_t schedule_entries(const CacheShape& s, int rows_of_a_tile) { return tiles_bound(s, rows_of_a_tile) + kTarget; }

// Before the parts of a large batch.
template <int ROWS>
void launch_schedule(const CacheAttendParams& P, hipStream_t stream) {
  if (P.s.B <= kWaveBatch) return;
  const int64_t entries = schedule_entries(P.s, ROWS), want = (entries + 4 * kScheduleThreads - 1) / (4 * kScheduleThreads);
  cache_schedule_kernel<ROWS><<<(unsigned)(want < 256 ? want : 256), kScheduleThreads, 0, stream>>>(P, (int)entries);
}

// Launches of the join, after the parts.
template <int D, int ROWS>
void launch_join(const CacheAttendParams& P, hipStream_t stream) {
  const int64_t all_rows = (int64_t)P.s.rows * P.s.G, all_tiles = tiles_bound(P.s, ROWS);
  const int rows = (int)(all_rows < ROWS ? all_rows : ROWS);             // of a tile
  const int tiles = (int)(all_tiles < kTarget ? all_tiles : kTarget);    // at most kTarget are split
  // from 64 tiles on most have few parts: at most 16 (kSlots / 64) on average, if all are split
  if (tiles < 64) {
    cache_join_kernel<D, ROWS><<<dim3(tiles, rows), 256, 0, stream>>>(P);
  } else {
    constexpr int per = 1024 / D;
    const int groups = (rows + per - 1) / per;
    const int each = ((rows < 16 ? rows : 16) + groups - 1) / groups;
    // (a part has min_pages at least)
    if (P.s.max_pages > kLongParts * P.min_pages)
      cache_join_rows_kernel<D, ROWS, true><<<dim3(tiles + kLongTiles * each, groups), 256, 0, stream>>>(P, tiles, each);
    else
      cache_join_rows_kernel<D, ROWS, false><<<dim3(tiles, groups), 256, 0, stream>>>(P, tiles, 0);
  }
}

}  // namespace
}  // namespace ugbs
