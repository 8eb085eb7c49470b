// Values that are not finite.
//
// A key that a row does not see has the probability 0, but in a tile that other rows do see it is multiplied like any other,
// and 0 times an infinity or NaN is NaN.  Tiles are not searched for such values: a row whose result comes out as NaN is
// computed once more here, from the keys that it sees alone, and is NaN only if it should be.  Nothing but the last check of
// the outputs is paid where all values are finite.  One wavefront does a row, with plain loads, 16 keys at a time.
#pragma once

#include "paged.h"

namespace heatkv {
namespace paged {

template <class T, bool FP8>
__device__ __forceinline__ float cache_value(const void* pages, long long at) {
  if constexpr (FP8)
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<const unsigned char*>(pages)[at], 0);
  else
    return static_cast<float>(static_cast<const T*>(pages)[at]);
}

// Query head hq of `token` over the granules [begin, end): locate(g) gives {row, pos, whether the row sees the granule's page}, keys
// from `limit` on are not seen.  probability(s): of a raw score, relative to the reference that the row's sum was formed with.
// store(column, value, sum of the probabilities) gets the unnormalised sums, two columns or one per lane.
template <class T, bool FP8, int D, class Locate, class Probability, class Store>
__device__ __forceinline__ void redo_row(const AttendParams& p, long long token, int hq, int limit, int begin, int end,
                                         const Locate& locate, const Probability& probability, const Store& store) {
  const int lane = threadIdx.x & 63, key = lane >> 2, quarter = lane & 3;
  const T* q = static_cast<const T*>(p.q.data) + token * p.q.token_stride + hq * p.q.head_stride;
  float x[D / 64] = {}, sum = 0.f;
  for (int g = begin; g < end && sum == sum; ++g) {  // behind a probability that is NaN everything stays NaN
    const auto at = locate(g);
    if (!at.seen || at.pos >= limit) continue;
    float s = 0.f;
    for (int i = quarter; i < D; i += 4)
      s = fmaf(static_cast<float>(q[i]), cache_value<T, FP8>(p.k_pages, (at.row + key) * D + i), s);
    s += __shfl_xor(s, 1, 64);
    s += __shfl_xor(s, 2, 64);
    const float e = at.pos + key < limit ? probability(s) : -1.f;
    for (int k = 0; k < 16; ++k) {
      const float w = __shfl(e, 4 * k, 64);
      if (!(w < 0.f)) {  // seen, whatever its probability
        sum += w;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) x[i] += w * cache_value<T, FP8>(p.v_pages, (at.row + k) * D + 64 * i + lane);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) store(64 * i + lane, x[i], sum);
}

struct RedoGranule {
  long long row;
  int pos;
  bool seen;
};

}  // namespace paged
}  // namespace heatkv
