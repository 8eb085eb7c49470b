// The paged cache (paged_*.hip): parameters of its kernels and what they share on the device.
//
// k_pages, v_pages [num_pages][H][page][d]; a request's token at position x lies in row x % page of page table[b][x / page].
// Pages are powers of two of 16 to 256 rows, so 16 rows from a position that is a multiple of 16 (a granule) are
// contiguous: the attention kernels take the cache granule by granule, each with one wavefront-uniform address.
//
// Lengths, tables and selections are device data that the host has not seen.  The kernels bring every number that becomes
// an address into its range first (one scalar instruction each): wrong tables give wrong outputs, not a fault.
#pragma once

#include <algorithm>

#include "device_util.h"

namespace heatkv {
namespace paged {

constexpr int GRANULE = 16;
constexpr int MAX_BATCH = 4096;

struct Cache {
  int H, G, Hq;  // kv heads, queries per kv head, H * G
  int page_log2, num_pages, batch, max_pages;
  int tokens;         // rows of the token tensors; those from q_start[batch] on belong to no request
  unsigned div_G;     // reciprocal of G, see divide()
  int causal;
  const int* table;   // [batch][max_pages]
  const int* q_start; // [batch + 1]
  const int* lens;    // [batch], new tokens among them
};

// n / d for n * d < 2^32 with the reciprocal floor(2^32 / d) + 1 (d > 1) or 0 (d = 1).
inline unsigned reciprocal(unsigned d) { return d > 1 ? static_cast<unsigned>((1ull << 32) / d + 1) : 0; }
__device__ __forceinline__ int divide(int n, unsigned recip) {
  return recip ? static_cast<int>(__umulhi(static_cast<unsigned>(n), recip)) : n;
}

// Scalar loads: the index is wavefront-uniform, the array is not written by the launch.
__device__ __forceinline__ int uniform_load(const int* p, long long i) {
  return ((const __attribute__((address_space(4))) int*)(p))[i];
}

// The largest b with first(q_start[b]) <= x, by one wavefront; first(q, b) grows with b.  Two rounds of loads side by side
// (up to 64 x 64 requests) instead of a chain of twelve.
template <class First>
__device__ __forceinline__ int find_request(const int* q_start, int batch, int x, int lane, First first) {
  int base = 0;
  if (batch > 64) {
    const int b = lane * 64;
    const bool below = b < batch && first(q_start[b], b) <= x;
    base = (max(__popcll(__ballot(below)), 1) - 1) * 64;
  }
  const int b = base + lane;
  const bool below = b < batch && first(q_start[b], b) <= x;
  return __builtin_amdgcn_readfirstlane(base + max(__popcll(__ballot(below)), 1) - 1);
}

// Tiles of ROWS query rows (token j, query g of the kv head's group: row j * G + g).  Requests have different numbers of
// new tokens, which the host does not know: request b's tiles are counted from (q_start[b] * G) / ROWS + b on, so that a
// tile's request follows from a search, and tokens * G / ROWS + batch tiles are enough; some are empty.
template <int ROWS>
__device__ __forceinline__ int first_tile(int q, int b, int G) { return q * G / ROWS + b; }
template <int ROWS>
inline int tile_count(int tokens, int G, int batch) { return static_cast<int>(static_cast<long long>(tokens) * G / ROWS) + batch; }

struct Tile {
  int b;          // request
  int q0, n_new;  // its first token, its new tokens
  int len;        // its keys
  int row0, rows; // first query row of the tile, rows of it that exist (<= 0: an empty tile)
};
__device__ __forceinline__ void fill_tile(const Cache& c, Tile& t) {
  const int q0 = uniform_load(c.q_start, t.b), q1 = uniform_load(c.q_start, t.b + 1);
  t.q0 = min(max(q0, 0), c.tokens);
  t.n_new = min(max(q1, t.q0), c.tokens) - t.q0;
  t.len = min(max(uniform_load(c.lens, t.b), 0), c.max_pages << c.page_log2);
}
template <int ROWS>
__device__ __forceinline__ Tile find_tile(const Cache& c, int tile, int lane) {
  Tile t;
  t.b = find_request(c.q_start, c.batch, tile, lane, [&](int q, int b) { return first_tile<ROWS>(min(max(q, 0), c.tokens), b, c.G); });
  fill_tile(c, t);
  t.row0 = (tile - first_tile<ROWS>(t.q0, t.b, c.G)) * ROWS;
  t.rows = t.row0 < 0 ? 0 : min(t.n_new * c.G - t.row0, ROWS);
  return t;
}
// Keys that token j of the request sees.
__device__ __forceinline__ int visible_keys(const Cache& c, const Tile& t, int j) {
  return c.causal ? max(t.len - t.n_new + j + 1, 0) : t.len;
}

// First row of a page of a kv head, in rows of the cache.
__device__ __forceinline__ long long page_row(const Cache& c, int entry, int h) {
  const unsigned e = min(static_cast<unsigned>(entry), static_cast<unsigned>(c.num_pages - 1));
  return (static_cast<long long>(e) * c.H + h) << c.page_log2;
}

// Exponent of the power of two that 8-bit codes count (page bounds, query codes): the least one with amax <= 127 * 2^e, and
// no less than -100, so that neither the power nor its inverse leaves the normal numbers.  amax <= 2^127.
__device__ __forceinline__ int code_exponent(float amax) {
  const float m = __builtin_amdgcn_frexp_mantf(amax);
  return amax > 0.f ? max(__builtin_amdgcn_frexp_expf(amax) - (m <= 127.f / 128.f ? 7 : 6), -100) : -100;
}

struct Rows {  // of the token tensors, strides in elements
  const void* data;
  long long token_stride, head_stride;
};

struct Border {
  int b, h, t, parts;  // a cut segment and its parts; 0: none at this workgroup
};

// Parts of cut segments: unnormalised outputs [..][ROWS][d], reference and sum [..][ROWS][2], two for each workgroup of the
// line, one for each that takes a piece.
struct Parts {
  float *o, *ml;
  Border* borders;  // of each workgroup; null: nothing can be cut
  int grid;         // workgroups of the launch; for the join, those that it looks at
};

struct AttendParams {
  Cache c;
  Rows q, out;
  const void *k_pages, *v_pages;
  const int* selected;  // [tokens][H][top], null: all pages
  int top;
  float sm_scale;
  float* lse;           // [tokens][Hq] or null
  // Requests of this launch, by their query rows per kv head (new tokens x group): least_rows < rows <= most_rows.
  int least_rows, most_rows;
  // How it is dealt (paged_schedule.h): shares, weight of the lightest one, segments from which on it goes another way.
  int workgroups, least_weight, whole_from;
  int cut_from;  // segments of up to this weight are not cut
  Parts parts;
};

// The launch's arguments, loaded anew.
__device__ __forceinline__ const AttendParams& arguments() {
  auto* at = (const __attribute__((address_space(4))) AttendParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("; arguments" : "+s"(at));
  return *(const AttendParams*)at;
}

struct SelectParams {
  Cache c, tokens_as_rows;  // the second with G = 1: tiles of tokens
  Rows q;
  const int8_t* bounds;      // [num_pages][H][2][d]
  const float* bound_scales; // [num_pages][H]
  int first, last, top, pitch;
  int* selected;             // [tokens][H][top]
};
constexpr size_t SELECT_LDS = 144 * 1024;  // what a workgroup may use: codes and scores of one token with 32768 pages

}  // namespace paged

using PagedSelectParams = paged::SelectParams;
using PagedAttendParams = paged::AttendParams;
using PagedParts = paged::Parts;
constexpr size_t PAGED_SELECT_LDS = paged::SELECT_LDS;
hipError_t launch_paged_select(const PagedSelectParams& p, int dtype, int d, hipStream_t stream);
hipError_t launch_paged_attend_bf16(const PagedAttendParams& p, int d, bool fp8, hipStream_t stream);
hipError_t launch_paged_attend_long(const PagedAttendParams& p, int d, bool fp8, hipStream_t stream);
hipError_t launch_paged_attend_f32(const PagedAttendParams& p, int d, hipStream_t stream);
// few, many: of the two attention launches, grid: join_workgroups(), 0 where there is nothing to join.
hipError_t launch_paged_join(const PagedAttendParams& p, const PagedParts& few, const PagedParts& many, int dtype, int d,
                             hipStream_t stream);

}  // namespace heatkv
