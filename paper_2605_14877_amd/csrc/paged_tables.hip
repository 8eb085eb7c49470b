// Paged cache: one step of the page allocator.  Block tables, the slots of the new tokens and the ring of free pages are
// brought forward from the requests' lengths, on the GPU: no length crosses to the host.
//
// Request b holds ceil(lens / page) pages and wants ceil((keep + new) / page).  Pages that it lacks come from the head of
// the ring, requests in order; pages that it no longer needs go behind the ring's tail, requests in order.  What is given
// back in a step is taken again in a later one at the earliest, so taking and giving never touch the same ring entry.
//
// Bound: latency, a chain of memory round trips (lengths; ring entries; table) and two block scans.  One workgroup does the
// request part; the slots come in the same launch where they are few, otherwise from a second one with a workgroup or
// more per request (a request's slots then need no search).
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

__global__ __launch_bounds__(LANES) void paged_assign_kernel(AssignArgs p, int slots_here) {
  __shared__ int take0[MAX_BATCH], give0[MAX_BATCH], q0[MAX_BATCH + 1];  // of every request: sums over those before it
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
    for (int w = 0; w < LANES / 64; ++w) {
      if (w < wave) before[k] += part[k][w];
      all[k] += part[k][w];
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

  // From here on nothing that a request's part reads is written by another one: lens_out may be lens, span_out span
  // (both have been read by every lane in front of the barrier above).
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    if (i < per && b < B) {
      take0[b] = static_cast<int>(before[0]);
      give0[b] = static_cast<int>(before[1]);
      q0[b] = ok ? static_cast<int>(before[2]) : 0;
      p.q_start[b] = q0[b];
      if (ok) {
        p.lens_out[b] = keep[i] + come[i];
      } else if (p.lens_out != p.lens) {
        p.lens_out[b] = p.lens[b];
      }
      before[0] += max(want(i) - held(i), 0);
      before[1] += max(held(i) - want(i), 0);
      before[2] += come[i];
    }
  }
  const int tokens = ok ? static_cast<int>(all[2]) : 0;
  if (tid == 0) {
    q0[B] = tokens;
    p.q_start[B] = tokens;
    p.status[0] = status;
    p.span_out[0] = ok ? static_cast<int>((head + all[0]) % R) : head;
    p.span_out[1] = ok ? static_cast<int>(count - all[0] + all[1]) : count;
  }
  __syncthreads();
  // Lengths of other lanes' requests, below: from keep and new_tokens, which nothing writes, and from the sums.
  if (ok) {
    const int takes = static_cast<int>(all[0]), gives = static_cast<int>(all[1]);
    auto pages_wanted = [&](int b) { return (p.keep[b] + p.new_tokens[b] + page - 1) >> lp; };
    for (int i = tid; i < takes; i += LANES) {
      const int b = find(take0, B, i);
      const int n = (b + 1 < B ? take0[b + 1] : takes) - take0[b];  // that the request takes: its last n pages
      const int entry = p.ring[(head + i) % R];
      p.table[static_cast<long long>(b) * p.max_pages + pages_wanted(b) - n + (i - take0[b])] = entry;
    }
    const long long tail = static_cast<long long>(head) + count;
    for (int i = tid; i < gives; i += LANES) {
      const int b = find(give0, B, i);
      p.ring[(tail + i) % R] = p.table[static_cast<long long>(b) * p.max_pages + pages_wanted(b) + (i - give0[b])];
    }
  }
  if (!slots_here) return;
  __syncthreads();  // the table entries written above, by this workgroup
  for (int t = tid; t < p.max_tokens; t += LANES) {
    int slot = -1;
    if (t < tokens) {
      const int b = find(q0, B, t);
      const int x = p.keep[b] + t - q0[b];
      slot = (p.table[static_cast<long long>(b) * p.max_pages + (x >> lp)] << lp) + (x & (page - 1));
    }
    p.slots[t] = slot;
  }
}

// Slots of request blockIdx.x's new tokens; blockIdx.x = batch: of the tokens that belong to no request.
__global__ __launch_bounds__(256) void paged_slots_kernel(AssignArgs p) {
  const int b = blockIdx.x, lp = p.page_log2, first = p.q_start[b];
  const int stop = b < p.batch ? p.q_start[b + 1] : static_cast<int>(p.max_tokens);
  const int keep = b < p.batch ? p.keep[b] : 0;
  for (int t = first + blockIdx.y * 256 + threadIdx.x; t < stop; t += gridDim.y * 256) {
    const int x = keep + t - first;
    p.slots[t] = b < p.batch ? (p.table[static_cast<long long>(b) * p.max_pages + (x >> lp)] << lp) + (x & ((1 << lp) - 1)) : -1;
  }
}

}  // namespace

hipError_t launch_paged_assign(const AssignArgs& a, hipStream_t stream) {
  const bool slots_here = a.max_tokens <= 4 * LANES;
  hipLaunchKernelGGL(paged_assign_kernel, dim3(1), dim3(LANES), 0, stream, a, slots_here ? 1 : 0);
  if (hipError_t e = hipGetLastError()) return e;
  if (slots_here) return hipSuccess;
  // workgroups enough to fill the chip however the tokens are spread over the requests
  const unsigned parts = static_cast<unsigned>(std::min<long long>((a.max_tokens + 255) / 256, std::max(1, 4096 / (a.batch + 1))));
  hipLaunchKernelGGL(paged_slots_kernel, dim3(a.batch + 1, parts), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace heatkv
