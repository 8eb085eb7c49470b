// Paged attention: joins the parts of segments that several workgroups had (paged_schedule.h).  A workgroup looks at one border
// between shares, or one piece, and joins the segment there if this is the first border in it, or its first piece: a wavefront
// per row, the parts in order, so that the result does not depend on which workgroup was done first.  One launch for both attention
// kernels.
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

// EACH: rows of a wavefront.  `set`: which 4 EACH rows of the segment.
template <class T, int D, int ROWS, int EACH>
__device__ __forceinline__ void join(const AttendParams& p, const Parts& from, int w, int set) {
  constexpr int N = D / 32;  // columns of a lane; either half of a wavefront has a whole row
  const int lane = threadIdx.x & 63, half = lane >> 5, col = (lane & 31) * N;
  const auto* at_border = (const __attribute__((address_space(4))) Border*)(from.borders) + w;
  const Border border{at_border->b, at_border->h, at_border->t, at_border->parts};
  const int parts = abs(border.parts);
  if (parts == 0) return;
  const Part segment{border.b, border.h, border.t, 0, 0, 0};
  const Tile tile = tile_of<ROWS>(p.c, segment);
  const int row0 = set * EACH * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // then every fourth
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
    y.m = from.ml[at * 2];
    y.l = from.ml[at * 2 + 1];
#pragma unroll
    for (int k = 0; k < N; ++k) y.x[k] = from.o[at * D + col + k];
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
          // Places behind the last part hold that part again: left out, not multiplied by 0, as it may hold infinities.
          const bool real = i0 + 2 * u < parts;
          const float g = factor(y[r][u].m, m);
          sum[r].l += g * (real ? y[r][u].l : 0.f);
#pragma unroll
          for (int k = 0; k < N; ++k) sum[r].x[k] += g * (real ? y[r][u].x[k] : 0.f);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r0 + 4 * r < tile.rows) finish(r0 + 4 * r, sum[r]);
  }
}

constexpr int FEW_EACH = 1, FEW_SETS = 16 / 4 / FEW_EACH, MANY_EACH = 4, MANY_SETS = 128 / 4 / MANY_EACH;

// 16 rows: the workgroups of one set are neighbours, so that with 8 kv heads a part is joined on the XCD that its workgroup ran on,
// out of its L2 (16 decoding requests 53.5 us, with the sets of a segment side by side 57).  128 rows: the sets side by side (whole
// scales 64 us, the other way 67).
// MANY: the 128-row kernel's as well (twice the registers, which cost a decoding step of 16 requests 4 us).
template <class T, int D, bool MANY>
__global__ __launch_bounds__(256) void paged_join_kernel(AttendParams p, Parts few, Parts many) {
  if constexpr (!MANY) return join<T, D, 16, FEW_EACH>(p, few, blockIdx.x, blockIdx.y);
  const int i = blockIdx.x, j = i - few.grid * FEW_SETS;
  if (j < 0) return join<T, D, 16, FEW_EACH>(p, few, i % few.grid, i / few.grid);
  if constexpr (MANY) join<T, D, 128, MANY_EACH>(p, many, j / MANY_SETS, j % MANY_SETS);
}

template <class T, int D, bool MANY = false>
hipError_t launch(const AttendParams& p, const Parts& few, const Parts& many, hipStream_t stream) {
  const dim3 grid = MANY ? dim3(few.grid * FEW_SETS + many.grid * MANY_SETS) : dim3(few.grid, FEW_SETS);
  hipLaunchKernelGGL((paged_join_kernel<T, D, MANY>), grid, dim3(256), 0, stream, p, few, many);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_join(const PagedAttendParams& p, const PagedParts& few, const PagedParts& many, int dtype, int d,
                             hipStream_t stream) {
  if (dtype == HEATKV_F32) return d == 128 ? launch<float, 128>(p, few, many, stream) : launch<float, 64>(p, few, many, stream);
  if (many.grid) return d == 128 ? launch<bf16_t, 128, true>(p, few, many, stream) : launch<bf16_t, 64, true>(p, few, many, stream);
  return d == 128 ? launch<bf16_t, 128>(p, few, many, stream) : launch<bf16_t, 64>(p, few, many, stream);
}

}  // namespace heatkv
