// Pages, slots and lengths of a step, from the requests' lengths and a stack
// of free pages.
//
// With held_b = ceil(ctx_b / 64) and need_b = ceil((ctx_b + new_b) / 64) -
// held_b, the requests' pages come off the stack in the order of the requests:
// with two prefix sums over the requests (pages given back, pages needed)
// every new page has a place of its own in the stack, so no workgroup waits for
// another: each one forms the sums for itself, and then takes its share of the
// slots.  Slot i of request b belongs to position ctx_b + i; the slot that
// begins a page also writes the table's entry.  Entries of a released request
// that are no page are not given back: where a request is released the others
// are counted first, 16 lanes to each (500 requests, 10 of them released: 8.5 -> 10.6 us).
#include "cache_internal.h"

namespace ugbs {
namespace {

constexpr int kThreads = 256;

struct PlanParams {
  CacheShape s;
  const int32_t* ctx_lens;
  const int32_t* new_lens;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* table;
  int32_t* kv_lens;
  int32_t* q_lens;
  int32_t* slots;
  int32_t* free_left;
};

struct Request {
  int ctx, q, held, need, back;   // cached tokens, tokens asked for (0: refused), pages held, needed, given back
  bool gone;                      // released
};

__device__ __forceinline__ Request request_of(const PlanParams& P, int b) {
  const int most = P.s.max_pages * kBlock;
  Request r;
  r.ctx = P.ctx_lens[b];
  const int n = P.new_lens[b];
  const bool sound = r.ctx >= 0 && r.ctx <= most;
  r.ctx = r.ctx < 0 ? 0 : r.ctx > most ? most : r.ctx;
  r.held = (r.ctx + kBlock - 1) / kBlock;
  r.gone = sound && n == UGBS_CACHE_RELEASE;
  r.back = r.gone ? r.held : 0;
  r.q = sound && n >= 0 && n <= P.s.rows && n <= most - r.ctx ? n : 0;
  r.need = (r.ctx + r.q + kBlock - 1) / kBlock - r.held;
  return r;
}

__device__ __forceinline__ bool is_page(const PlanParams& P, int32_t x) { return x >= 0 && x < P.s.n_pages; }

__global__ void __launch_bounds__(kThreads) cache_plan_kernel(PlanParams P) {
  extern __shared__ int s_sum[];            // [B] pages given back before request b, [B] needed before it
  __shared__ int s_wave[2][kThreads / 64];
  __shared__ int s_gone, s_holes;           // released requests; entries of theirs that are no page
  const int B = P.s.B, tid = threadIdx.x;
  int* const s_back = s_sum;
  int* const s_need = s_sum + B;
  const int per = (B + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, B), b1 = min(b0 + per, B);
  const int count = P.free_count[0];
  int back = 0, need = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    const Request r = request_of(P, b);
    s_back[b] = r.back;
    back += r.back;
    need += r.need;
  }
  if (tid == 0) s_gone = s_holes = 0;
  if (__syncthreads_or(back > 0)) {
    for (int b = b0; b < b1; ++b)
      if (s_back[b] > 0) s_need[atomicAdd(&s_gone, 1)] = b;       // (in any order)
    __syncthreads();
    for (int k = tid / 16; k < s_gone; k += kThreads / 16) {
      const int b = s_need[k], n = s_back[b];
      const int32_t* const row = P.table + (size_t)b * P.s.max_pages;
      int c = 0;
      for (int p = tid % 16; p < n; p += 8 * 16) {
        int32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = row[min(p + 16 * i, n - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) c += p + 16 * i < n && is_page(P, x[i]);
      }
#pragma unroll
      for (int o = 1; o < 16; o *= 2) c += __shfl_xor(c, o);
      if (tid % 16 == 0 && c < n) {
        s_back[b] = c;
        s_holes = 1;
      }
    }
    __syncthreads();
    back = 0;
    for (int b = b0; b < b1; ++b) back += s_back[b];
  }
  const int back_in = scan_add(back), need_in = scan_add(need);
  const int w = tid >> 6;
  if ((tid & 63) == 63) {
    s_wave[0][w] = back_in;
    s_wave[1][w] = need_in;
  }
  __syncthreads();
  int back_at = back_in - back, need_at = need_in - need, back_all = 0;
#pragma unroll
  for (int v = 0; v < kThreads / 64; ++v) {
    if (v < w) {
      back_at += s_wave[0][v];
      need_at += s_wave[1][v];
    }
    back_all += s_wave[0][v];
  }
  const int held0 = min(max(count, 0), P.s.n_pages);
  const int stock = min(held0 + back_all, P.s.n_pages);      // free pages to take from
  int taken = 0;                                             // pages granted up to this thread's last request
  for (int b = b0; b < b1; ++b) {
    const Request r = request_of(P, b);
    const int r_back = s_back[b];
    s_back[b] = back_at;
    s_need[b] = need_at;
    const bool ok = r.need == 0 || need_at + r.need <= stock;
    if (ok && r.need > 0) taken = need_at + r.need;
    if (blockIdx.x == 0) {
      P.kv_lens[b] = r.gone ? 0 : r.ctx + (ok ? r.q : 0);
      P.q_lens[b] = ok ? r.q : 0;
    }
    back_at += r_back;
    need_at += r.need;
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    // the granted requests that need pages are the first ones: the most pages taken
#pragma unroll
    for (int o = 1; o < 64; o *= 2) taken = max(taken, __shfl_xor(taken, o));
    if ((tid & 63) == 0) s_wave[1][w] = taken;
    __syncthreads();
    if (tid == 0) {
      for (int v = 1; v < kThreads / 64; ++v) taken = max(taken, s_wave[1][v]);
      P.free_left[0] = stock - taken;
    }
  }
  // the page at place j of the pages given back
  auto returned = [&](int j) -> int32_t {
    int lo = 0, hi = B - 1;                 // the last request with s_back[b] <= j
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_back[mid] <= j) lo = mid;
      else hi = mid - 1;
    }
    const int32_t* const row = P.table + (size_t)lo * P.s.max_pages;
    int k = j - s_back[lo];
    if (!s_holes) return row[k];
#pragma unroll 1
    for (int p = 0; p < P.s.max_pages; p += 16) {
      int32_t x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = row[min(p + i, P.s.max_pages - 1)];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (p + i < P.s.max_pages && is_page(P, x[i]) && k-- == 0) return x[i];
    }
    return -1;
  };
  const int stride = gridDim.x * kThreads, first = blockIdx.x * kThreads + tid;
  for (int j = first; j < stock - held0; j += stride) P.free_pages[held0 + j] = returned(j);
  // four slots a thread at a time, so that their loads are on their way together
  const int rows = P.s.rows, total = B * rows;
  for (int base = blockIdx.x * 4 * kThreads + tid; base < total; base += 4 * stride) {
    int place[4], from[4], page[4];
    bool new_page[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(base + k * kThreads, total - 1), b = at / rows, i = at - b * rows;
      const Request r = request_of(P, b);
      const int pos = r.ctx + i, p = pos / kBlock;
      place[k] = i < r.q && (r.need == 0 || s_need[b] + r.need <= stock) ? pos : -1;
      from[k] = stock - 1 - s_need[b] - (p - r.held);
      new_page[k] = p >= r.held;
      page[k] = -1;
      if (place[k] >= 0) {
        if (!new_page[k]) page[k] = P.table[(size_t)b * P.s.max_pages + p];
        else page[k] = from[k] >= held0 ? returned(from[k] - held0) : P.free_pages[from[k]];
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = base + k * kThreads;
      if (at >= total) break;
      if (place[k] >= 0 && new_page[k] && place[k] % kBlock == 0)
        P.table[(size_t)(at / rows) * P.s.max_pages + place[k] / kBlock] = page[k];
      // an entry that is no page gives no slot
      P.slots[at] = place[k] >= 0 && is_page(P, page[k]) ? page[k] * kBlock + place[k] % kBlock : -1;
    }
  }
}

}  // namespace

hipError_t launch_cache_plan(const CacheShape& s, const int32_t* ctx_lens, const int32_t* new_lens, int32_t* free_pages,
                             const int32_t* free_count, int32_t* table, int32_t* kv_lens, int32_t* q_lens, int32_t* slots,
                             int32_t* free_left, hipStream_t stream) {
  const PlanParams P{s, ctx_lens, new_lens, free_pages, free_count, table, kv_lens, q_lens, slots, free_left};
  const int64_t items = (int64_t)s.B * s.rows;
  const int64_t want = (items + 4 * kThreads - 1) / (4 * kThreads);
  const unsigned grid = (unsigned)(want < 1024 ? want : 1024);
  cache_plan_kernel<<<grid, kThreads, 2 * sizeof(int) * s.B, stream>>>(P);
  return hipGetLastError();
}

}  // namespace ugbs
