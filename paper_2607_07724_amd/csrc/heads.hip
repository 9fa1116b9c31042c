// A projection's rows as queries, keys and values by heads: [B, rows, heads, d] with any
// strides to [B, heads, rows, d], the norm of each query and key head and its rotation by
// position on the way.  One pass: every number is read once and written once.
#include "heads_internal.h"

namespace ugbs {
namespace {

constexpr int kWaves = 4, kTokenWaves = 1;

template <int D, int PAIRS>
__global__ void __launch_bounds__(64 * kWaves) heads_split_kernel(HeadsParams P, int heads_each) {
  __shared__ __align__(16) float2 s_angle[kTokenWaves * kTokens<D> * D / 2];
  const int h0 = blockIdx.y * heads_each, all = P.s.H + 2 * P.s.Hkv;
  split_heads<D, PAIRS, kWaves, kTokenWaves>(P, place_in_row(blockIdx.x, gridDim.x) * (kTokenWaves * kTokens<D>), h0, min(h0 + heads_each, all), s_angle);
}

template <int D, int PAIRS>
void split(const HeadsParams& P, hipStream_t stream) {
  constexpr int T = kTokenWaves * kTokens<D>;
  const int64_t groups = ((int64_t)P.s.B * P.s.rows + T - 1) / T;
  const int heads = P.s.H + 2 * P.s.Hkv, slices = head_slices(groups, heads, kWaves / kTokenWaves), each = (heads + slices - 1) / slices;
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
