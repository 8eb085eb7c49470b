// Paged attention: joins the parts of segments that lie in several workgroups' shares (paged_schedule.h).  A workgroup looks at
// one border between shares and joins the segment there, if this is the first border in it: a wavefront per row, the parts in
// order, so that the result does not depend on which workgroup was done first.
//
// Bound: latency (three rounds of loads, and one more for every sixteen parts), and of many rows the traffic of the parts.
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
  constexpr int N = D / 32, U = 8;  // columns of a lane, parts whose loads a half wavefront has under way together
  const int lane = threadIdx.x & 63, w = blockIdx.x + 1;
  const auto* border = (const __attribute__((address_space(4))) Border*)(p.borders) + w;
  const int parts = border->parts;
  if (parts == 0) return;
  const Part segment{border->b, border->h, border->t, 0, 0, 0};
  const Tile tile = tile_of<ROWS>(p.c, segment);
  const f32m::Exponent prob(p.sm_scale);
  const float c = p.sm_scale * kLog2e;
  for (int i = 0; i < EACH; ++i) {
  const int row = (blockIdx.y * EACH + i) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= tile.rows) return;
  auto place = [&](int i) { return part_rows<ROWS>(w - 1 + i, i == 0) + row; };
  float m = -INFINITY;
  for (int i = lane; i < parts; i += 64) m = fmaxf(m, p.part_ml[place(i) * 2]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d, 64));
  float l = 0.f, x[N] = {};
  const int half = lane >> 5, col = (lane & 31) * N;
  for (int i0 = half; i0 < parts; i0 += 2 * U) {  // the halves take turns
    float ml[U][2], o[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at_row = place(min(i0 + 2 * u, parts - 1));
      ml[u][0] = p.part_ml[at_row * 2];
      ml[u][1] = p.part_ml[at_row * 2 + 1];
#pragma unroll
      for (int k = 0; k < N; ++k) o[u][k] = p.part_o[at_row * D + col + k];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 2 * u >= parts) break;
      const float f = sizeof(T) == 4 ? prob(ml[u][0], m) : fast_exp2((ml[u][0] - m) * c);
      l += f * ml[u][1];
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] += f * o[u][k];
    }
  }
  l += swap_halves(l);
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] += swap_halves(x[k]);
  const float f = l > 0.f ? 1.f / l : l;  // nothing seen: zeros; NaN stays
  const int j = divide(tile.row0 + row, p.c.div_G), hq = segment.h * p.c.G + tile.row0 + row - j * p.c.G;
  const long long t = tile.q0 + j;
  T* to = static_cast<T*>(const_cast<void*>(p.out.data)) + t * p.out.token_stride + hq * p.out.head_stride + col;
  if (half == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = static_cast<T>(x[k] * f);
  if (p.lse && lane == 0) p.lse[t * p.c.Hq + hq] = sizeof(T) == 4 ? natural_lse_f32(m, l, prob) : natural_lse(m, l, p.sm_scale);
  }
}

template <class T, int D, int ROWS, int EACH>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((paged_join_kernel<T, D, ROWS, EACH>), dim3(p.workgroups - 1, ROWS / 4 / EACH), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_join(const PagedAttendParams& p, int dtype, int d, bool many, hipStream_t stream) {
  if (dtype == HEATKV_F32) return d == 128 ? launch<float, 128, 16, 1>(p, stream) : launch<float, 64, 16, 1>(p, stream);
  if (many) return d == 128 ? launch<bf16_t, 128, 128, 8>(p, stream) : launch<bf16_t, 64, 128, 8>(p, stream);
  return d == 128 ? launch<bf16_t, 128, 16, 1>(p, stream) : launch<bf16_t, 64, 16, 1>(p, stream);
}

}  // namespace heatkv
