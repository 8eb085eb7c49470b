// Paged cache: one step of the page allocator.  Block tables, the slots of the new tokens and the ring of free pages are
// brought forward from the requests' lengths, on the GPU: no length crosses to the host.
//
// Request b holds ceil(lens / page) pages and wants ceil((keep + new) / page).  Pages that it lacks come from the head of
// the ring, requests in order; pages that it no longer needs go behind the ring's tail, requests in order.  What is given
// back in a step is taken again in a later one at the earliest, so taking and giving never touch the same ring entry.
//
// Bound: latency, a chain of memory round trips (lengths; ring or table entries) and a block scan.  Small steps are one
// workgroup.  In larger ones every workgroup makes the scan for itself and moves its share of pages and slots; as lens_out
// and span_out may be lens and span, which all of them read, these are written by a second launch, which scans once more (also
// where they are arrays of their own).
// 1024 requests, finished ones replaced by new prompts: 13.7 us, by one workgroup 84; 64 decoding requests: 7.1 us by one workgroup,
// 11 by two launches.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "paged.h"

namespace heatkv {

namespace {

using namespace paged;

constexpr int LANES = 1024;
constexpr int PER_LANE = MAX_BATCH / LANES;

__device__ __forceinline__ long long wave_scan(long long v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long long u = __shfl_up(v, d, 64);
    if (lane >= d) v += u;
  }
  return v;
}

// Largest b in [0, n) with first[b] <= x; first[0] = 0, ascending.
__device__ __forceinline__ int find(const int* first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    (first[mid] <= x ? lo : hi) = mid;
  }
  return lo;
}

// MOVE: pages, slots, q_start and status, shared by the grid's workgroups.  COMMIT: lens_out and span_out, by workgroup 0,
// which is the only one if there is MOVE as well.
template <bool MOVE, bool COMMIT>
__global__ __launch_bounds__(LANES) void paged_assign_kernel(AssignArgs p) {
  __shared__ int take0[MOVE ? MAX_BATCH : 1], give0[MOVE ? MAX_BATCH : 1], q0[MOVE ? MAX_BATCH : 1];  // sums over the requests before
  __shared__ long long part[3][LANES / 64];
  __shared__ int any_bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int B = p.batch, R = p.num_pages, lp = p.page_log2, page = 1 << lp;
  if (tid == 0) any_bad = 0;
  __syncthreads();
  const int head = p.span[0], count = p.span[1];

  int len[PER_LANE], keep[PER_LANE], come[PER_LANE];
  long long sum[3] = {0, 0, 0};  // pages to take, pages to give, tokens: of this lane's requests
  bool bad = false;
  const long long most = static_cast<long long>(p.max_pages) << lp;
  const int per = (B + LANES - 1) / LANES;  // requests per lane, consecutive ones
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    len[i] = keep[i] = come[i] = 0;
    if (i < per && b < B) {
      len[i] = p.lens[b];
      keep[i] = p.keep[b];
      come[i] = p.new_tokens[b];
      if (len[i] < 0 || len[i] > most || keep[i] < 0 || keep[i] > len[i] || come[i] < 0 ||
          static_cast<long long>(keep[i]) + come[i] > most) {
        bad = true;
        len[i] = keep[i] = come[i] = 0;
      }
    }
  }
  auto held = [&](int i) { return (len[i] + page - 1) >> lp; };
  auto want = [&](int i) { return (keep[i] + come[i] + page - 1) >> lp; };
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    sum[0] += max(want(i) - held(i), 0);
    sum[1] += max(held(i) - want(i), 0);
    sum[2] += come[i];
  }
  long long before[3], all[3] = {0, 0, 0};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const long long inc = wave_scan(sum[k], lane);
    before[k] = inc - sum[k];
    if (lane == 63) part[k][wave] = inc;
  }
  if (bad) any_bad = 1;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) {
      const long long x = part[k][w];
      if (w < wave) before[k] += x;
      all[k] += x;
    }
  int status = HEATKV_PAGED_OK;
  if (any_bad)
    status = HEATKV_PAGED_BAD_LENGTH;
  else if (head < 0 || head >= R || count < 0 || count > R || count + all[1] > R)
    status = HEATKV_PAGED_BAD_FREE_LIST;
  else if (all[2] > p.max_tokens)
    status = HEATKV_PAGED_TOO_MANY_TOKENS;
  else if (all[0] > count)
    status = HEATKV_PAGED_NO_PAGES;
  const bool ok = status == HEATKV_PAGED_OK;
  const int takes = ok ? static_cast<int>(all[0]) : 0, gives = ok ? static_cast<int>(all[1]) : 0;
  const int tokens = ok ? static_cast<int>(all[2]) : 0;
  const bool first_group = blockIdx.x == 0;

  // Where this workgroup is the only one, it has read lens and span to the end (the barrier above): they may be the outputs.
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    if (i < per && b < B) {
      if constexpr (MOVE) {
        take0[b] = static_cast<int>(before[0]);
        give0[b] = static_cast<int>(before[1]);
        q0[b] = static_cast<int>(before[2]);
        if (first_group) p.q_start[b] = ok ? static_cast<int>(before[2]) : 0;
        before[0] += max(want(i) - held(i), 0);
        before[1] += max(held(i) - want(i), 0);
        before[2] += come[i];
      }
      if constexpr (COMMIT) {
        if (ok)
          p.lens_out[b] = keep[i] + come[i];
        else if (p.lens_out != p.lens)
          p.lens_out[b] = p.lens[b];
      }
    }
  }
  if (tid == 0 && first_group) {
    if constexpr (MOVE) {
      p.q_start[B] = tokens;
      p.status[0] = status;
    }
    if constexpr (COMMIT) {
      const int next = head + takes;  // both below 2^26
      p.span_out[0] = ok ? next < R ? next : next - R : head;
      p.span_out[1] = ok ? count - takes + gives : count;
    }
  }
  if constexpr (!MOVE) return;
  __syncthreads();

  // Requests other than the lane's own, below: from keep and new_tokens, which nothing writes, and from the sums.
  const int at = blockIdx.x * LANES + tid, stride = gridDim.x * LANES;
  auto wanted = [&](int b) { return (p.keep[b] + p.new_tokens[b] + page - 1) >> lp; };
  auto row = [&](int b) { return p.table + static_cast<long long>(b) * p.max_pages; };
  auto taken = [&](int i) { return p.ring[head + i < R ? head + i : head + i - R]; };
  auto takes_of = [&](int b) { return (b + 1 < B ? take0[b + 1] : takes) - take0[b]; };
  for (int i = at; i < takes; i += stride) {
    const int b = find(take0, B, i);
    row(b)[wanted(b) - takes_of(b) + i - take0[b]] = taken(i);  // the last pages of the request
  }
  const unsigned tail = static_cast<unsigned>(head) + count;  // below 2 R, i below R
  for (int i = at; i < gives; i += stride) {
    const int b = find(give0, B, i);
    unsigned to = tail + i;
    to -= to >= static_cast<unsigned>(R) ? R : 0;
    to -= to >= static_cast<unsigned>(R) ? R : 0;
    p.ring[to] = row(b)[wanted(b) + i - give0[b]];
  }
  for (int t = at; t < p.max_tokens; t += stride) {
    int slot = -1;
    if (t < tokens) {
      const int b = find(q0, B, t);
      const int x = p.keep[b] + t - q0[b], i = x >> lp, n = takes_of(b), old = wanted(b) - n;
      // the table's new entries may be another workgroup's to write
      const int entry = n > 0 && i >= old ? taken(take0[b] + i - old) : row(b)[i];
      slot = (entry << lp) + (x & (page - 1));
    }
    p.slots[t] = slot;
  }
}

}  // namespace

hipError_t launch_paged_assign(const AssignArgs& a, hipStream_t stream) {
  if (a.max_tokens <= 2 * LANES && a.batch <= 128) {
    hipLaunchKernelGGL((paged_assign_kernel<true, true>), dim3(1), dim3(LANES), 0, stream, a);
    return hipGetLastError();
  }
  const unsigned groups = static_cast<unsigned>(std::min<long long>((a.max_tokens + LANES - 1) / LANES + a.batch / 32, 128));
  hipLaunchKernelGGL((paged_assign_kernel<true, false>), dim3(groups), dim3(LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((paged_assign_kernel<false, true>), dim3(1), dim3(LANES), 0, stream, a);
  return hipGetLastError();
}

}  // namespace heatkv
