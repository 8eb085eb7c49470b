// The keys that a tile of 16 query rows walks over, in granules of 16 and steps of two granules: all pages of the request, or
// the union of the pages that the tile's tokens have chosen, with the tokens that chose each.
#pragma once

#include <atomic>

#include "f32_mfma.h"
#include "paged.h"

namespace heatkv {
namespace paged {

constexpr size_t WALK_LDS = 144 * 1024;

// Where 16 consecutive keys lie.  pos: position of the first one; `row`, in rows of the cache, is in range also for granules
// behind the walk's end, whose position no row sees.
struct Granule {
  long long row;
  int pos;
  unsigned tokens;  // chosen pages: bit i = the tile's token i reads the page
};

// V stage of a wavefront: 32 rows of d bf16 elements, in windows of 32 bytes; the merge parks 16 x (d + 4) floats in it.
constexpr int stage_bytes(int d) { return 16 * (d + 4) * 4; }
template <int D>
__device__ __forceinline__ int stage_swizzle(int row) { return D == 128 ? row & 7 : (row >> 1) & 3; }

inline int walk_capacity(const AttendParams& p) {  // pages that a tile's tokens can have chosen between them
  const long long tokens = std::min(16, 15 / p.c.G + 2);
  return static_cast<int>(std::min<long long>(p.c.max_pages, tokens * p.top));
}
inline size_t walk_lds_bytes(const AttendParams& p) {
  return 16 + (p.c.max_pages + 31) / 32 * 8 + static_cast<size_t>(walk_capacity(p)) * 8;
}

// before[i] = bits set in the words in front of word i; returns how many there are.  By one wavefront.
__device__ __forceinline__ int scan_bits(const unsigned* bits, int* before, int words, int lane) {
  int sum = 0;
  for (int i = lane; i - lane < words; i += 64) {
    const int n = i < words ? __popc(bits[i]) : 0;
    int inc = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int u = __shfl_up(inc, d, 64);
      if (lane >= d) inc += u;
    }
    if (i < words) before[i] = sum + inc - n;
    sum += __shfl(inc, 63, 64);
  }
  return sum;
}

// Pages that the tokens of a tile of 128 rows can have chosen between them.
__device__ __forceinline__ int many_capacity(const Cache& c, int top) {
  return static_cast<int>(min(static_cast<long long>(c.max_pages), static_cast<long long>(min(128, 127 / c.G + 2)) * top));
}

template <bool CHOSEN>
struct Walk;

template <>
struct Walk<false> {
  const Cache& c;
  const int h;
  const long long table;
  const int granules;
  __device__ __forceinline__ Walk(const AttendParams& p, const Tile& t, int head, int, int, int limit_max, char*, int)
      : c(p.c), h(head), table(static_cast<long long>(t.b) * p.c.max_pages), granules((limit_max + GRANULE - 1) / GRANULE) {}
  __device__ __forceinline__ int steps() const { return (granules + 1) / 2; }
  __device__ __forceinline__ Granule locate(int granule) const {
    const int x = min(granule, granules - 1) * GRANULE;
    return {page_row(c, uniform_load(c.table, table + (x >> c.page_log2)), h) + (x & ((1 << c.page_log2) - 1)),
            granule * GRANULE, 0};
  }
  __device__ __forceinline__ bool sees(const Granule&, int) const { return true; }
};

template <>
struct Walk<true> {
  const Cache& c;
  const int h;
  const long long table;
  const int *pages, *tokens;  // LDS: the union in ascending order, who chose each
  int n_pages;
  // By all lanes of the workgroup (256).
  __device__ __forceinline__ Walk(const AttendParams& p, const Tile& t, int head, int j_first, int j_last, int limit_max,
                                  char* lds, int tid)
      : c(p.c), h(head), table(static_cast<long long>(t.b) * p.c.max_pages) {
    const int words = (c.max_pages + 31) / 32;
    int* const count = reinterpret_cast<int*>(lds);
    unsigned* const bits = reinterpret_cast<unsigned*>(lds + 16);
    int* const before = reinterpret_cast<int*>(bits + words);
    int* const list = before + words;
    const int capacity = min(c.max_pages, min(16, 15 / c.G + 2) * p.top);
    unsigned* const who = reinterpret_cast<unsigned*>(list + capacity);
    for (int i = tid; i < words; i += 256) bits[i] = 0;
    for (int i = tid; i < capacity; i += 256) who[i] = 0;
    __syncthreads();
    const int seen = (limit_max + (1 << c.page_log2) - 1) >> c.page_log2;
    const int entries = (j_last - j_first + 1) * p.top;
    // token i's choices lie H * top apart
    auto entry = [&](int i, int& token) {
      token = i / p.top;
      const int x = p.selected[((static_cast<long long>(t.q0) + j_first + token) * c.H + h) * p.top + i - token * p.top];
      return x < seen ? x : -1;
    };
    for (int i = tid; i < entries; i += 256) {
      int token;
      const int x = entry(i, token);
      if (x >= 0) atomicOr(&bits[x >> 5], 1u << (x & 31));
    }
    __syncthreads();
    if (tid < 64) {
      const int total = scan_bits(bits, before, words, tid);
      if (tid == 0) *count = total;
    }
    __syncthreads();
    for (int i = tid; i < entries; i += 256) {
      int token;
      const int x = entry(i, token);
      if (x >= 0) {
        const int at = before[x >> 5] + __popc(bits[x >> 5] & ((1u << (x & 31)) - 1));
        list[at] = x;
        atomicOr(&who[at], 1u << token);
      }
    }
    __syncthreads();
    pages = list;
    tokens = reinterpret_cast<const int*>(who);
    n_pages = __builtin_amdgcn_readfirstlane(*count);
  }
  __device__ __forceinline__ int steps() const { return ((n_pages << (c.page_log2 - 4)) + 1) / 2; }
  __device__ __forceinline__ Granule locate(int granule) const {
    const int per = c.page_log2 - 4, u = min(granule >> per, n_pages - 1), off = (granule & ((1 << per) - 1)) * GRANULE;
    const int x = __builtin_amdgcn_readfirstlane(pages[u]);
    const unsigned who = (granule >> per) < n_pages ? __builtin_amdgcn_readfirstlane(tokens[u]) : 0;
    return {page_row(c, uniform_load(c.table, table + x), h) + off, (x << c.page_log2) + off, who};
  }
  __device__ __forceinline__ bool sees(const Granule& at, int token) const { return at.tokens >> token & 1; }
};

// Natural logarithm of a row's sum of exponentials: reference m in units of the raw scores, l = sum 2^((s - m) c).
__device__ __forceinline__ float natural_lse(float m, float l, float sm_scale) {
  return l > 0.f ? fmaf(m, sm_scale, 0.6931471805599453f * __builtin_amdgcn_logf(l)) : l == 0.f ? -INFINITY : l;
}
// The same of the fp32 kernels: reference and exponents as f32m::Exponent has them, l = 2^-8 of the sum.
__device__ __forceinline__ float natural_lse_f32(float m, float l, const f32m::Exponent& prob) {
  return l > 0.f ? 0.6931471805599453f * fmaf(m, prob.up, __builtin_amdgcn_logf(l) + 8.f) : l == 0.f ? -INFINITY : l;
}

// Raises a kernel's limit of dynamic LDS on the current device, once; not an operation of the stream, so a capture does not
// mind.  `done`: one bit per device ordinal below 64.
inline hipError_t allow_lds(const void* kernel, size_t bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  if (dev >= 0 && dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return hipSuccess;
  if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes))) return e;
  if (dev >= 0 && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return hipSuccess;
}

}  // namespace paged
}  // namespace heatkv
