// Attention of new tokens over the paged cache, few query rows per request: the kernel of its own (paged_attend_few.h says how it goes).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "paged_attend_few.h"

namespace heatkv {

namespace {

using namespace paged;

extern __shared__ __attribute__((aligned(16))) char paged_lds[];

template <int D, Format F, bool CHOSEN>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void paged_attend_kernel(AttendParams p) {
  __shared__ FewShared shared;
  attend_few<D, F, CHOSEN, 0>(p, blockIdx.x, shared, paged_lds, paged_lds + FEW_WAVES * stage_bytes(D));
}

template <int D, Format F, bool CHOSEN>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  const size_t lds = FEW_WAVES * stage_bytes(D) + (CHOSEN ? walk_lds_bytes(p) : 0);
  static std::atomic<unsigned long long> allowed{0};
  if (lds > 64 * 1024)
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(&paged_attend_kernel<D, F, CHOSEN>), WALK_LDS, allowed)) return e;
  hipLaunchKernelGGL((paged_attend_kernel<D, F, CHOSEN>), dim3(p.parts.grid), dim3(64 * FEW_WAVES), lds, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attend_bf16(const PagedAttendParams& p, int d, int kv_format, hipStream_t stream) {
  auto run = [&](auto d_tag, auto chosen) {
    constexpr int D = decltype(d_tag)::value;
    constexpr bool CHOSEN = decltype(chosen)::value;
    return kv_format == HEATKV_KV_FP4_E2M1   ? launch<D, E2M1, CHOSEN>(p, stream)
           : kv_format == HEATKV_KV_FP8_E4M3 ? launch<D, E4M3, CHOSEN>(p, stream)
                                             : launch<D, NATIVE, CHOSEN>(p, stream);
  };
  using D128 = std::integral_constant<int, 128>;
  using D64 = std::integral_constant<int, 64>;
  if (p.selected) return d == 128 ? run(D128{}, std::true_type{}) : run(D64{}, std::true_type{});
  return d == 128 ? run(D128{}, std::false_type{}) : run(D64{}, std::false_type{});
}

}  // namespace heatkv
