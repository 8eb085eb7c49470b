// Values that are not finite.
//
// A key that a row does not see has the probability 0, but in a tile that other rows do see it is multiplied like any other,
// and 0 times an infinity or NaN is NaN.  Tiles are not searched for such values: a row whose result comes out as NaN is
// looked at once more here, by one wavefront, with plain loads.  Nothing but the last check of the outputs is paid where all
// values are finite.
//
// Over all pages, the keys that a row does not see follow those that it sees, within the last tiles.  Where their values are finite
// the NaN is the row's own and stays: a few keys are read instead of all.  Otherwise, and of chosen pages always, the NaN columns
// are computed anew from the keys that the row sees, 16 at a time, until each is NaN or the keys are through.  300 new tokens x 4
// heads over 4096 keys, d = 128, one NaN in V: 41 us where all rows see it (36 without; 2400 with all rows done anew key by key),
// 430 among the new tokens, 1000 in the last one; on a page that some of 1024 tokens have chosen: 2600 (142 without).
#pragma once

#include "paged.h"

namespace heatkv {
namespace paged {

template <class T, Format F, int D>
__device__ __forceinline__ float cache_value(const void* pages, long long row, int col) {
  if constexpr (F == E4M3) {
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<const unsigned char*>(pages)[row * D + col], 0);
  } else if constexpr (F == E2M1) {
    const int r = static_cast<int>(row) & 15;
    const auto* at = static_cast<const unsigned char*>(pages) + (row - r) * row_bytes<T, F>(D);
    const unsigned code = at[r * (D / 2) + col / 2] >> (col & 1 ? 4 : 0);
    return static_cast<float>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale_of(at[8 * D + r * (D / 32) + col / 32]), 0)[0]);
  } else {
    return static_cast<float>(static_cast<const T*>(pages)[row * D + col]);
  }
}

// Query head hq of `token` over the granules [begin, end): locate(g) gives {row, pos, whether the row sees the granule's page}, keys
// from `limit` on are not seen, and none of those from `len` on was read.  probability(s): of a raw score, relative to the reference
// that the row's sum was formed with.  stored(column): the result so far; store(column, value, sum of the probabilities) gets the
// unnormalised sums of the columns that were NaN.  with_sum: the row's sum is wrong as well, and formed to its end; returns it.
template <class T, Format F, int D, bool CHOSEN, class Locate, class Probability, class Stored, class Store>
__device__ __forceinline__ float redo_row(const AttendParams& p, long long token, int hq, int limit, int len, int begin, int end,
                                          bool with_sum, const Locate& locate, const Probability& probability, const Stored& stored,
                                          const Store& store) {
  constexpr int N = D / 64;  // columns of a lane
  const int lane = threadIdx.x & 63, key = lane >> 2, quarter = lane & 3;
  bool nan[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = stored(64 * i + lane);
    nan[i] = y != y;
  }
  if constexpr (!CHOSEN) {
    bool reached = false;
    for (int g = max(begin, limit >> 4); g < end && !reached; ++g) {
      const auto at = locate(g);
      if (at.pos >= len) break;
      for (int k = max(limit - at.pos, 0); k < min(len - at.pos, 16); ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float v = cache_value<T, F, D>(p.v_pages, at.row + k, 64 * i + lane);
          reached = reached || (nan[i] && !(fabsf(v) < INFINITY));
        }
      reached = __any(reached);
    }
    if (!reached) return 0.f;
  }
  const T* q = static_cast<const T*>(p.q.data) + token * p.q.token_stride + hq * p.q.head_stride;
  float x[N] = {}, sum = 0.f;
  for (int g = begin; g < end && sum == sum; ++g) {  // behind a probability that is NaN everything stays NaN
    const auto at = locate(g);
    if (!at.seen || at.pos >= limit) continue;
    float v[16][N];  // all loads of a granule under way together; of keys that the row does not see not used
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) v[k][i] = cache_value<T, F, D>(p.v_pages, at.row + k, 64 * i + lane);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D; i += 4)
      s = fmaf(static_cast<float>(q[i + quarter]), cache_value<T, F, D>(p.k_pages, at.row + key, i + quarter), s);
    s += __shfl_xor(s, 1, 64);
    s += __shfl_xor(s, 2, 64);
    const float e = at.pos + key < limit ? probability(s) : -1.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), 4 * k));
      if (!(w < 0.f)) {  // seen, whatever its probability
        sum += w;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += w * v[k][i];
      }
    }
    bool open = with_sum;
#pragma unroll
    for (int i = 0; i < N; ++i) open = open || (nan[i] && x[i] == x[i]);
    if (!__any(open)) break;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (nan[i]) store(64 * i + lane, x[i], sum);
  return sum;
}

struct RedoGranule {
  long long row;
  int pos;
  bool seen;
};

}  // namespace paged
}  // namespace heatkv
