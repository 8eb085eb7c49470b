// Paged attention: joins the parts of segments that several workgroups had (paged_schedule.h).  A workgroup looks at one border
// between shares, or one piece, and joins the segment there if this is the first border in it, or its first piece: a wavefront
// per row, the parts in order, so that the result does not depend on which workgroup was done first.
//
// Bound: latency (borders, lengths, parts: a round of loads each, one more for every sixteen parts), and of many rows the
// traffic of the parts.  4 to 5 us; 500 pieces of 128 rows, d = 128 (33 MB): 13 us.  Four rows to a wavefront there: with
// eight it takes 2 us longer, with two 1 to 2 us less, but 3 us more where there is nothing to join.
#include <hip/hip_runtime.h>

#include "f32_mfma.h"
#include "kernels.h"
#include "paged.h"
#include "paged_schedule.h"
#include "paged_walk.h"

namespace heatkv {

namespace {

using namespace paged;

// EACH: rows of a wavefront.
template <class T, int D, int ROWS, int EACH>
__global__ __launch_bounds__(256) void paged_join_kernel(AttendParams p) {
  constexpr int N = D / 32;  // columns of a lane; either half of a wavefront has a whole row
  const int lane = threadIdx.x & 63, half = lane >> 5, col = (lane & 31) * N, w = blockIdx.x;
  const auto* at_border = (const __attribute__((address_space(4))) Border*)(p.borders) + w;
  const Border border{at_border->b, at_border->h, at_border->t, at_border->parts};
  const int parts = abs(border.parts);
  if (parts == 0) return;
  const Part segment{border.b, border.h, border.t, 0, 0, 0};
  const Tile tile = tile_of<ROWS>(p.c, segment);
  const int row0 = blockIdx.y * EACH * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // then every fourth
  if (row0 >= tile.rows) return;
  const f32m::Exponent prob(p.sm_scale);
  const float c = p.sm_scale * kLog2e;
  // 2^ of a difference of references.
  auto factor = [&](float reference, float to) { return sizeof(T) == 4 ? prob(reference, to) : fast_exp2((reference - to) * c); };
  struct One {
    float m, l, x[N];
  };
  auto load = [&](int part, int row) {
    const long long at = joined_rows<ROWS>(border, w, part, p.c.H) + row;
    One y;
    y.m = p.part_ml[at * 2];
    y.l = p.part_ml[at * 2 + 1];
#pragma unroll
    for (int k = 0; k < N; ++k) y.x[k] = p.part_o[at * D + col + k];
    return y;
  };
  // What the two halves have of a row becomes the output.
  auto finish = [&](int row, One y) {
    const float m = max_halves(y.m), f = factor(y.m, m);
    const float l = sum_halves(y.l * f), g = l > 0.f ? 1.f / l : l;  // nothing seen: zeros; NaN stays
    const int j = divide(tile.row0 + row, p.c.div_G), hq = segment.h * p.c.G + tile.row0 + row - j * p.c.G;
    const long long t = tile.q0 + j;
    T* to = static_cast<T*>(const_cast<void*>(p.out.data)) + t * p.out.token_stride + hq * p.out.head_stride + col;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float x = sum_halves(y.x[k] * f) * g;
      if (half == 0) to[k] = static_cast<T>(x);
    }
    if (p.lse && lane == 0) p.lse[t * p.c.Hq + hq] = sizeof(T) == 4 ? natural_lse_f32(m, l, prob) : natural_lse(m, l, p.sm_scale);
  };
  if (parts == 2) {  // the loads of all rows together
    One y[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) y[i] = load(half, min(row0 + 4 * i, tile.rows - 1));
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (row0 + 4 * i < tile.rows) finish(row0 + 4 * i, y[i]);
    return;
  }
  // R rows and of each U parts have their loads under way together; the halves take turns over the parts.
  constexpr int R = EACH < 4 ? EACH : 4, U = 8 / (R < 2 ? 1 : 2);
  for (int r0 = row0; r0 < min(row0 + 4 * EACH, tile.rows); r0 += 4 * R) {
    One sum[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = One{-INFINITY, 0.f, {}};
    for (int i0 = half; i0 - half < parts; i0 += 2 * U) {
      One y[R][U];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < U; ++u) y[r][u] = load(min(i0 + 2 * u, parts - 1), min(r0 + 4 * r, tile.rows - 1));
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float m = sum[r].m;
#pragma unroll
        for (int u = 0; u < U; ++u) m = fmaxf(m, y[r][u].m);
        const float f = factor(sum[r].m, m);
        sum[r].m = m;
        sum[r].l *= f;
#pragma unroll
        for (int k = 0; k < N; ++k) sum[r].x[k] *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float g = i0 + 2 * u < parts ? factor(y[r][u].m, m) : 0.f;
          sum[r].l += g * y[r][u].l;
#pragma unroll
          for (int k = 0; k < N; ++k) sum[r].x[k] += g * y[r][u].x[k];
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r0 + 4 * r < tile.rows) finish(r0 + 4 * r, sum[r]);
  }
}

template <class T, int D, int ROWS, int EACH>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((paged_join_kernel<T, D, ROWS, EACH>), dim3(p.grid, ROWS / 4 / EACH), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_join(const PagedAttendParams& p, int dtype, int d, bool many, hipStream_t stream) {
  if (dtype == HEATKV_F32) return d == 128 ? launch<float, 128, 16, 1>(p, stream) : launch<float, 64, 16, 1>(p, stream);
  if (many) return d == 128 ? launch<bf16_t, 128, 128, 4>(p, stream) : launch<bf16_t, 64, 128, 4>(p, stream);
  return d == 128 ? launch<bf16_t, 128, 16, 1>(p, stream) : launch<bf16_t, 64, 16, 1>(p, stream);
}

}  // namespace heatkv
