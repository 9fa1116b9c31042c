// A projection's rows as queries, keys and values by heads: [B, rows, heads, d] with any
// strides to [B, heads, rows, d], the norm of each query and key head and its rotation by
// position on the way.  One pass: every number is read once and written once, so HBM bounds it
// where tokens are many, with reads and writes in equal parts: 32K tokens of 28/4 heads, d 128 (604 MB) 113 us,
// 5.3 TB/s.  A wave has one head of the tokens of its workgroup at a time (kTokens), the next one's rows
// on their way.  1, 2, 8 or 16 waves a workgroup for 4 changed nothing (123 to 126 us before stores passed
// the caches and each XCD had its tokens in a row, 113 since).
#include "heads_internal.h"

namespace ugbs {
namespace {

constexpr int kWaves = 4;

template <int D, int PAIRS>
__global__ void __launch_bounds__(64 * kWaves) heads_split_kernel(HeadsParams P, int heads_each) {
  __shared__ __align__(16) float2 s_angle[kTokens<D> * D / 2];
  const int h0 = blockIdx.y * heads_each, all = P.s.H + 2 * P.s.Hkv;
  split_heads<D, PAIRS, kWaves>(P, place_in_row(blockIdx.x, gridDim.x) * kTokens<D>, h0, min(h0 + heads_each, all), s_angle);
}

template <int D, int PAIRS>
void split(const HeadsParams& P, hipStream_t stream) {
  constexpr int T = kTokens<D>;
  const int64_t groups = ((int64_t)P.s.B * P.s.rows + T - 1) / T;
  const int heads = P.s.H + 2 * P.s.Hkv, slices = head_slices(groups, heads, kWaves), each = (heads + slices - 1) / slices;
  heads_split_kernel<D, PAIRS><<<dim3((unsigned)groups, (heads + each - 1) / each), 64 * kWaves, 0, stream>>>(P, each);
}

template <int D>
void split(const HeadsParams& P, hipStream_t stream) {
  (P.s.pairs == UGBS_HALVES ? split<D, UGBS_HALVES> : split<D, UGBS_NEIGHBOURS>)(P, stream);
}

}  // namespace

hipError_t launch_heads_split(const HeadsParams& P, hipStream_t stream) {
  if (P.s.d == 64) split<64>(P, stream);
  else if (P.s.d == 128) split<128>(P, stream);
  else split<256>(P, stream);
  return hipGetLastError();
}

}  // namespace ugbs
