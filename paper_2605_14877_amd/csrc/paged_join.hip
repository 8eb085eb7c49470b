// Paged attention: joins the parts of rows whose keys were split over workgroups.  A wavefront per row and query head, the
// parts in order: the result does not depend on which workgroup was done first.
//
// Bound: latency of the few rows that are split at all (launches that do not fill the chip without).
#include <hip/hip_runtime.h>

#include "f32_mfma.h"
#include "kernels.h"
#include "paged.h"
#include "paged_walk.h"

namespace heatkv {

namespace {

using namespace paged;

template <class T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(AttendParams p) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const long long row = static_cast<long long>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= p.part_rows) return;
  // Token and query head of the row, if it is one (its entry of `parts` has no value otherwise).
  int t, h;
  if (p.short_requests) {
    const int kv = static_cast<int>(row % p.c.H), in = static_cast<int>(row / p.c.H % LONG_ROWS);
    Tile tile;
    tile.b = static_cast<int>(row / p.c.H / LONG_ROWS);
    fill_tile(p.c, tile);
    if (in >= tile.n_new * p.c.G || tile.n_new * p.c.G > LONG_ROWS) return;
    const int j = divide(in, p.c.div_G);
    t = tile.q0 + j;
    h = kv * p.c.G + in - j * p.c.G;
  } else {
    t = static_cast<int>(row / p.c.Hq);
    h = static_cast<int>(row - static_cast<long long>(t) * p.c.Hq);
    if (t >= uniform_load(p.c.q_start, p.c.batch)) return;
    if (p.long_only) {  // the long kernel's requests
      const int b = find_request(p.c.q_start, p.c.batch, t, lane, [](int q, int) { return q; });
      Tile tile;
      tile.b = b;
      fill_tile(p.c, tile);
      if (tile.n_new * p.c.G <= LONG_ROWS) return;
    }
  }
  const int parts = min(uniform_load(p.parts, row), p.splits);
  if (parts <= 1) return;
  const float* ml = p.part_ml + row * 2;
  float m = ml[0];
  for (int s = 1; s < parts; ++s) m = fmaxf(m, ml[s * p.part_rows * 2]);
  float l = 0.f, x[N] = {};
  const f32m::Exponent prob(p.sm_scale);
  const float c = p.sm_scale * kLog2e;
  for (int s = 0; s < parts; ++s) {
    const float d = ml[s * p.part_rows * 2];
    const float f = sizeof(T) == 4 ? prob(d, m) : fast_exp2((d - m) * c);
    l += f * ml[s * p.part_rows * 2 + 1];
    const float* o = p.part_o + (s * p.part_rows + row) * D + lane * N;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += f * o[i];
  }
  const float f = l > 0.f ? 1.f / l : l;
  T* to = static_cast<T*>(const_cast<void*>(p.out.data)) + t * p.out.token_stride + h * p.out.head_stride + lane * N;
#pragma unroll
  for (int i = 0; i < N; ++i) to[i] = static_cast<T>(x[i] * f);
  if (p.lse && lane == 0) p.lse[static_cast<long long>(t) * p.c.Hq + h] = sizeof(T) == 4 ? natural_lse_f32(m, l, prob) : natural_lse(m, l, p.sm_scale);
}

}  // namespace

hipError_t launch_paged_join(const PagedAttendParams& p, int dtype, int d, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((p.part_rows + 3) / 4)), block(256);
  if (dtype == HEATKV_F32) {
    if (d == 128)
      hipLaunchKernelGGL((paged_join_kernel<float, 128>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((paged_join_kernel<float, 64>), grid, block, 0, stream, p);
  } else {
    if (d == 128)
      hipLaunchKernelGGL((paged_join_kernel<bf16_t, 128>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((paged_join_kernel<bf16_t, 64>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace heatkv
