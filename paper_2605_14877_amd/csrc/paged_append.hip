// Paged cache: the rows of new tokens into their slots, and the 8-bit bounds of the keys on every page that they touch.
//
// Bounds of a page and kv head, over its valid rows: per channel the largest key value and minus the smallest one, as
// whole numbers of a power of two 2^e that is common to the page, rounded upwards: codes[0][d], codes[1][d] (int8).  e is
// the least exponent with which the largest magnitude fits 127 times.  Largest and smallest values are exact, multiplying by
// a power of two is exact, so the codes do not depend on the order of anything: the same bits whichever kernel forms them.
// Infinities and values beyond count as +-2^127, NaN as 0: a bound is always a number.
//
// Bound: memory traffic for prompts (rows in, rows out, 16 bytes per lane), latency for single tokens.  A page's bounds are
// formed anew from all of its valid rows, which costs a decoding step up to a page of older rows per head, but needs no
// running state that would have to follow when tokens are dropped or pages change owners.  12 prompts, 12000 tokens, 8 heads, d =
// 128, into 8-bit pages: 73.5 MB in 21 us, 3.5 TB/s; the rows alone take 13 us.  4-bit pages, without bounds: 11820 tokens,
// 61 MB, 12.9 us, 4.8 TB/s, and back as values 13.3 us.  Rows moved, 65900 of bf16: 540 MB in 84 to 94 us, 5.7 to 6.4 TB/s.
#include <type_traits>

#include "copy_rows.h"
#include "kernels.h"
#include "paged.h"

namespace heatkv {

namespace {

using paged::E2M1;
using paged::E4M3;
using paged::Format;
using paged::NATIVE;

constexpr int LANES = 256;
// Tokens x heads up to which a workgroup takes a page, so that its rows are read by 256 lanes; a wavefront beyond.  A token each,
// 8 heads, pages of 16, 64, 256 rows: 32 requests 4.5, 4.8, 6.7 us by workgroups, 4.7, 5.4, 10.4 by wavefronts; 128 requests
// 6.3, 7.0, 10.9 and 4.8, 6.5, 12.2; 512 requests, pages of 64, 17.2 and 13.9.
constexpr long long FEW_PAGES = 512;

// 8 values of a row, as floats.
template <class T>
__device__ __forceinline__ void values8(const uint4 (&raw)[sizeof(T) / 2], float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const unsigned w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  } else {
    const unsigned w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// 4-bit rows.  8 channels of a row are a lane's, so a block of 32 is four lanes next to one another, which are always all at work.
__device__ __forceinline__ unsigned max_of_four(unsigned x) {
  auto swapped = [](unsigned y, auto control) {
    return static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(y), decltype(control)::value, 0xf, 0xf, true));
  };
  x = max(x, swapped(x, std::integral_constant<int, 0xb1>{}));  // lanes 1, 0, 3, 2
  return max(x, swapped(x, std::integral_constant<int, 0x4e>{}));  // lanes 2, 3, 0, 1
}
// Codes of 8 bf16 values and the scale byte of their block: the power of two 2^e with the least e that the largest magnitude
// fits 7 times (it is then rounded by half a step at most, as the others are), -100 <= e <= 125; 255 if there is a NaN.
// The bits of a magnitude (1 + m / 128) 2^x are 128 (x + 127) + m: e = x - 2 up to m = 96, x - 1 beyond.
__device__ __forceinline__ uint2 nibbles_of(const uint4& raw) {
  const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
  unsigned most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
  most = max_of_four(most);
  const int byte = most > 0x7f80u ? 255 : min(max(static_cast<int>((most + 31) >> 7) - 2, 27), 252);
  const float scale = paged::scale_of(byte);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
  return make_uint2(c, byte);
}

// 8 values of a cache row as it is stored: raw[0].x, .y for 8 codes of 8 bits, for 8 of 4 bits and their scale byte.  `at`: row
// of the cache * D + column.
template <class T, Format F, int D>
struct CacheEight {
  static constexpr int N = sizeof(T) / 2;
  uint4 raw[N];
  struct Nibbles {
    long long codes, scale;
  };
  static __device__ __forceinline__ Nibbles nibbles_at(long long at) {
    const int r = static_cast<int>(at / D) & 15, col = static_cast<int>(at) & (D - 1);
    const long long granule = at / (16 * D) * (16 * paged::row_bytes<T, F>(D));
    return {granule + r * (D / 2) + col / 2, granule + 8 * D + r * (D / 32) + col / 32};
  }
  __device__ __forceinline__ void load(const void* pages, long long at) {
    if constexpr (F == E2M1) {
      const Nibbles n = nibbles_at(at);
      raw[0].x = *reinterpret_cast<const unsigned*>(static_cast<const char*>(pages) + n.codes);
      raw[0].y = static_cast<const unsigned char*>(pages)[n.scale];
    } else if constexpr (F == E4M3) {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const char*>(pages) + at);
      raw[0].x = w.x;
      raw[0].y = w.y;
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) raw[j] = ldg16(static_cast<const T*>(pages) + at + 4 * j);
    }
  }
  __device__ __forceinline__ void store(void* pages, long long at) const {
    if constexpr (F == E2M1) {
      const Nibbles n = nibbles_at(at);
      *reinterpret_cast<unsigned*>(static_cast<char*>(pages) + n.codes) = raw[0].x;
      if ((at & 31) == 0) static_cast<unsigned char*>(pages)[n.scale] = static_cast<unsigned char>(raw[0].y);
    } else if constexpr (F == E4M3) {
      *reinterpret_cast<uint2*>(static_cast<char*>(pages) + at) = make_uint2(raw[0].x, raw[0].y);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) *reinterpret_cast<uint4*>(static_cast<T*>(pages) + at + 4 * j) = raw[j];
    }
  }
  // From values as the operands have them.
  __device__ __forceinline__ void encode() {
    if constexpr (F == E2M1) {
      const uint2 c = nibbles_of(raw[0]);
      raw[0].x = c.x;
      raw[0].y = c.y;
    } else if constexpr (F == E4M3) {
      const uint2 c = make_uint2(bf16x4_to_e4m3(raw[0].x, raw[0].y), bf16x4_to_e4m3(raw[0].z, raw[0].w));
      raw[0].x = c.x;
      raw[0].y = c.y;
    }
  }
  // The values, as the operands have them.
  __device__ __forceinline__ void decode(uint4 (&x)[N]) const {
    if constexpr (F == E2M1)
      x[0] = __builtin_bit_cast(uint4, paged::nibbles_to_bf16(raw[0].x, paged::scale_of(raw[0].y)));
    else if constexpr (F == E4M3)
      x[0] = __builtin_bit_cast(uint4, paged::codes_to_bf16(raw[0].x, raw[0].y));
    else
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = raw[j];
  }
};

// A lane's token, head and place within the row, of PIECES; heads of a token are neighbours.  Tokens x heads are at most 2^23.
struct RowPiece {
  unsigned t;
  int h, piece;
};
template <int PIECES>
__device__ __forceinline__ RowPiece row_piece(int H) {
  const unsigned i = blockIdx.x * LANES + threadIdx.x, row = i / PIECES, t = row / static_cast<unsigned>(H);
  return {t, static_cast<int>(row - t * H), static_cast<int>(i % PIECES)};
}
// Row of the cache that slot has for head h.
template <class Args>
__device__ __forceinline__ long long cache_row(const Args& p, int slot, int h) {
  return ((static_cast<long long>(slot >> p.page_log2) * p.H + h) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
}
template <class Args>
__device__ __forceinline__ bool in_cache(const Args& p, int slot) {
  return static_cast<unsigned>(slot) < static_cast<unsigned>(p.num_pages << p.page_log2);
}

// Where new rows come from, columns col .. col + 7 of head h: the caller's token tensors, in the operands' type, or (MOVE) other rows of
// the cache, as they are.
template <class T, Format F, int D, bool MOVE>
struct Incoming {
  const PagedAppendArgs& p;
  const int h, col;
  const T *k_new, *v_new;
  __device__ __forceinline__ Incoming(const PagedAppendArgs& args, int head, int column)
      : p(args), h(head), col(column),
        k_new(MOVE ? nullptr : static_cast<const T*>(args.k_new) + head * args.k_head_stride + column),
        v_new(MOVE ? nullptr : static_cast<const T*>(args.v_new) + head * args.v_head_stride + column) {}
  __device__ __forceinline__ void fetch(long long t, CacheEight<T, F, D>& k, CacheEight<T, F, D>& v) const {  // row t of the call
    if constexpr (MOVE) {
      const unsigned slot = min(static_cast<unsigned>(p.from[t]), static_cast<unsigned>((p.num_pages << p.page_log2) - 1));
      const long long at = cache_row(p, static_cast<int>(slot), h) * D + col;
      k.load(p.k_pages, at);
      v.load(p.v_pages, at);
    } else {
      const T *kp = k_new + t * p.k_token_stride, *vp = v_new + t * p.v_token_stride;
#pragma unroll
      for (int j = 0; j < static_cast<int>(sizeof(T)) / 2; ++j) {
        k.raw[j] = ldg16(kp + 4 * j);
        v.raw[j] = ldg16(vp + 4 * j);
      }
    }
  }
};
// Into the cache; k is what the cache then holds.
template <bool MOVE, class Eight>
__device__ __forceinline__ void write_row(const PagedAppendArgs& p, long long at, Eight& k, Eight& v) {
  if constexpr (!MOVE) {
    k.encode();
    v.encode();
  }
  k.store(p.k_pages, at);
  v.store(p.v_pages, at);
}

// Rows only: 8 elements of K and of V per lane.
template <class T, Format F, int D>
__global__ __launch_bounds__(LANES) void paged_append_kernel(PagedAppendArgs p) {
  const RowPiece x = row_piece<D / 8>(p.H);
  if (x.t >= p.tokens) return;
  const int slot = p.slots[x.t];
  if (!in_cache(p, slot)) return;
  CacheEight<T, F, D> k, v;
  Incoming<T, F, D, false>(p, x.h, 8 * x.piece).fetch(x.t, k, v);
  write_row<false>(p, cache_row(p, slot, x.h) * D + 8 * x.piece, k, v);
}

// Rows moved as they are, without bounds: 16 bytes of K and of V per lane; of a 4-bit row the scale bytes of K by its first lane, those
// of V by its second.
template <class T, Format F, int D>
__global__ __launch_bounds__(LANES) void paged_move_kernel(PagedAppendArgs p) {
  constexpr int BYTES = F == E2M1 ? D / 2 : paged::row_bytes<T, F>(D), GRANULE_BYTES = 16 * paged::row_bytes<T, F>(D);
  const RowPiece x = row_piece<BYTES / 16>(p.H);
  if (x.t >= p.tokens) return;
  const int slot = p.slots[x.t];
  if (!in_cache(p, slot)) return;
  const int from_slot = static_cast<int>(min(static_cast<unsigned>(p.from[x.t]), static_cast<unsigned>((p.num_pages << p.page_log2) - 1)));
  const long long from = cache_row(p, from_slot, x.h), to = cache_row(p, slot, x.h);
  auto at = [&](long long row) {
    return (row >> 4) * GRANULE_BYTES + (row & 15) * BYTES + 16 * x.piece;  // codes of 16 rows lie together
  };
  char *const kp = static_cast<char*>(p.k_pages), *const vp = static_cast<char*>(p.v_pages);
  const uint4 k = ldg16(kp + at(from)), v = ldg16(vp + at(from));
  if constexpr (F == E2M1) {
    using Scales = std::conditional_t<D == 128, unsigned, unsigned short>;
    auto scales_at = [&](long long row) { return (row >> 4) * GRANULE_BYTES + 8 * D + (row & 15) * (D / 32); };
    char* const pages = x.piece == 0 ? kp : vp;
    if (x.piece < 2) *reinterpret_cast<Scales*>(pages + scales_at(to)) = *reinterpret_cast<const Scales*>(pages + scales_at(from));
  }
  *reinterpret_cast<uint4*>(kp + at(to)) = k;
  *reinterpret_cast<uint4*>(vp + at(to)) = v;
}

// The first token of a call on a page is that page's owner: who has it forms the bounds over the rows up to the last one that
// the call brings to the page (tokens of one page follow one another, as the allocator hands out slots).

// Codes of a page and head from the largest and minus the smallest values of columns 8 c .. 8 c + 7, on lane c of COLS (the
// other lanes of the wavefront have the same again).
template <int D>
__device__ __forceinline__ void store_bounds(const PagedAppendArgs& p, long long at, int lane, const float (&top)[8],
                                             const float (&low)[8]) {
  constexpr int COLS = D / 8;
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fmaxf(fabsf(top[i]), fabsf(low[i])));
#pragma unroll
  for (int m = 1; m < COLS; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
  const int e = paged::code_exponent(amax);
  auto code = [&](float x) {
    const int c = static_cast<int>(ceilf(ldexpf(x, -e)));
    return static_cast<int8_t>(c == 0 && x > 0.f ? 1 : c);  // upwards also where the quotient underflows
  };
  if (lane < COLS) {
    union {
      int8_t c[8];
      uint2 w;
    } a, b;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a.c[i] = code(top[i]);
      b.c[i] = code(low[i]);
    }
    *reinterpret_cast<uint2*>(p.bounds + at * (2 * D) + 8 * lane) = a.w;
    *reinterpret_cast<uint2*>(p.bounds + at * (2 * D) + D + 8 * lane) = b.w;
  }
  if (lane == 0) p.bound_scales[at] = ldexpf(1.f, e);
}
// Largest and smallest values of 8 columns over a lane's rows.  Infinities stay what they are until the end; whether there
// was a NaN is only noticed, and the rows are then gone through again by fold().
// bf16 values (8-bit codes are turned into such): as 16-bit whole numbers of the same order, two to an instruction, 2.5
// instructions a value.  fp32: 3 a value.  With NaN and range looked after for every value it was 7, and the kernel of many
// pages bound by that.
typedef short s16x2 __attribute__((ext_vector_type(2)));
template <class T>
struct Extremes {
  s16x2 top[4], low[4];
  __device__ __forceinline__ Extremes() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      top[i] = s16x2{-32768, -32768};
      low[i] = s16x2{32767, 32767};
    }
  }
  static __device__ __forceinline__ s16x2 ordered(unsigned w) {
    const s16x2 x = __builtin_bit_cast(s16x2, w);
    return x ^ ((x >> 15) & s16x2{0x7fff, 0x7fff});  // its own inverse
  }
  __device__ __forceinline__ void add(const uint4 (&raw)[1]) {
    const unsigned w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const s16x2 x = ordered(w[i]);
      top[i] = __builtin_elementwise_max(top[i], x);
      low[i] = __builtin_elementwise_min(low[i], x);
    }
  }
  // The largest values and minus the smallest ones, of no rows -inf; whether there was a NaN.
  __device__ __forceinline__ bool finish(float (&t)[8], float (&l)[8]) const {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const short a = top[i >> 1][i & 1], b = low[i >> 1][i & 1];
      const bool none = a < b;
      nan = nan || (!none && (a > 0x7f80 || b < static_cast<short>(0x807f)));
      auto value = [](short x) { return __uint_as_float(static_cast<unsigned>(static_cast<unsigned short>(x ^ ((x >> 15) & 0x7fff))) << 16); };
      t[i] = none ? -INFINITY : fminf(fmaxf(value(a), -0x1p127f), 0x1p127f);
      l[i] = none ? -INFINITY : fminf(fmaxf(-value(b), -0x1p127f), 0x1p127f);
    }
    return nan;
  }
};
template <>
struct Extremes<float> {
  float top[8], low[8], sum = 0.f;
  __device__ __forceinline__ Extremes() {
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = low[i] = -INFINITY;
  }
  __device__ __forceinline__ void add(const uint4 (&raw)[2]) {
    float x[8];
    values8<float>(raw, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      top[i] = fmaxf(top[i], x[i]);
      low[i] = fmaxf(low[i], -x[i]);
      sum = fmaf(x[i], 0.f, sum);  // NaN from a NaN on, and from an infinity
    }
  }
  __device__ __forceinline__ bool finish(float (&t)[8], float (&l)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool none = top[i] == -INFINITY && low[i] == -INFINITY;
      t[i] = none ? -INFINITY : fminf(fmaxf(top[i], -0x1p127f), 0x1p127f);
      l[i] = none ? -INFINITY : fminf(fmaxf(low[i], -0x1p127f), 0x1p127f);
    }
    return sum != sum;
  }
};
__device__ __forceinline__ void fold(const float (&x)[8], float (&top)[8], float (&low)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = x[i] == x[i] ? fminf(fmaxf(x[i], -0x1p127f), 0x1p127f) : 0.f;
    top[i] = fmaxf(top[i], y);
    low[i] = fmaxf(low[i], -y);
  }
}
template <int COLS>
__device__ __forceinline__ void fold_rows(float (&top)[8], float (&low)[8]) {  // over the rows of a wavefront
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int m = COLS; m < 64; m *= 2) {
      top[i] = fmaxf(top[i], __shfl_xor(top[i], m, 64));
      low[i] = fmaxf(low[i], __shfl_xor(low[i], m, 64));
    }
}
template <class T, Format F, int D>
__device__ __forceinline__ void add_to(Extremes<T>& e, const CacheEight<T, F, D>& x) {
  uint4 w[sizeof(T) / 2];
  x.decode(w);
  e.add(w);
}
// The rare case: rows [r0, rows) in steps of `step`, one by one, from the cache.
template <class T, Format F, int D>
__device__ __forceinline__ void fold_with_nan(const void* pages, long long base, int r0, int step, int rows, float (&top)[8],
                                              float (&low)[8]) {
  float t[8], l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = l[i] = -INFINITY;
  for (int r = r0; r < rows; r += step) {
    CacheEight<T, F, D> k;
    k.load(pages, base + r * D);
    uint4 raw[sizeof(T) / 2];
    k.decode(raw);
    float x[8];
    values8<T>(raw, x);
    fold(x, t, l);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top[i] = t[i];
    low[i] = l[i];
  }
}

// Few pages: a workgroup per token and head; those that own a page write its new rows and read the older ones.
template <class T, Format F, int D, bool MOVE>
__global__ __launch_bounds__(LANES) void paged_append_bounds_kernel(PagedAppendArgs p) {
  constexpr int COLS = D / 8, ROWS = LANES / COLS;  // lanes of a row, rows side by side
  constexpr int U = 4;                              // rows of a lane whose loads are under way together
  __shared__ float part[LANES / 64][2][D];
  __shared__ int run_end[LANES / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = blockIdx.x / p.H, h = blockIdx.x - t * p.H, lp = p.page_log2, page = 1 << lp;
  const int slots_all = p.num_pages << lp;
  const int s0 = paged::uniform_load(p.slots, t), prev = t > 0 ? paged::uniform_load(p.slots, t - 1) : -1;
  if (s0 < 0 || s0 >= slots_all) return;
  const int o0 = s0 & (page - 1);
  if (o0 != 0 && prev == s0 - 1) return;
  // n: end of the run of consecutive slots within the page (at most as many rows as there are lanes)
  const bool in_run = tid < page - o0 && t + tid < p.tokens && p.slots[t + tid] == s0 + tid;
  const unsigned long long missing = __ballot(!in_run);
  if (lane == 0) run_end[wave] = missing ? 64 * wave + __builtin_ctzll(missing) : page;
  __syncthreads();
  int n = page - o0;
#pragma unroll
  for (int w = 0; w < LANES / 64; ++w) n = min(n, run_end[w]);
  const int rows = o0 + n, col = (tid % COLS) * 8, r0 = tid / COLS;
  const long long at = static_cast<long long>(s0 >> lp) * p.H + h, base = (at << lp) * D + col;
  const Incoming<T, F, D, MOVE> incoming(p, h, col);
  Extremes<T> seen;
  for (int first = r0; first < rows; first += ROWS * U) {
    CacheEight<T, F, D> k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = first + ROWS * u;
      if (r >= rows) continue;
      if (r < o0)
        k[u].load(p.k_pages, base + r * D);
      else
        incoming.fetch(t + r - o0, k[u], v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = first + ROWS * u;
      if (r >= rows) continue;
      if (r >= o0) write_row<MOVE>(p, base + r * D, k[u], v[u]);
      add_to(seen, k[u]);
    }
  }
  float top[8], low[8];
  if (seen.finish(top, low)) {
    if constexpr (F == E2M1) __threadfence_block();  // scale bytes that the lane next to it has written
    fold_with_nan<T, F, D>(p.k_pages, base, r0, ROWS, rows, top, low);  // its own rows, written above
  }
  fold_rows<COLS>(top, low);
  if (lane < COLS)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      part[wave][0][col + i] = top[i];
      part[wave][1][col + i] = low[i];
    }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 1; w < LANES / 64; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      top[i] = fmaxf(top[i], part[w][0][col + i]);
      low[i] = fmaxf(low[i], part[w][1][col + i]);
    }
  store_bounds<D>(p, at, lane, top, low);
}

// Many pages: a wavefront per page, without barriers.  It looks for owners among `chunk` tokens (at most 64) of one kv head, and
// its first rows are under way before it knows how many count.  Rows first and the bounds by a second launch, which reads them
// back, took 13.5 + 13 us; this takes 21.
template <class T, Format F, int D, bool MOVE>
__global__ __launch_bounds__(LANES) void paged_append_pages_kernel(PagedAppendArgs p, int chunk) {
  constexpr int COLS = D / 8, ROWS = 64 / COLS, U = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the heads of a token next to one another: their rows are neighbours in memory
  const int group = blockIdx.x / p.H, h = blockIdx.x - group * p.H, lp = p.page_log2, page = 1 << lp;
  const long long t0 = (static_cast<long long>(group) * (LANES / 64) + wave) * chunk;
  const int slots_all = p.num_pages << lp;
  auto slot_of = [&](long long t) {
    const int s = t >= 0 && t < p.tokens ? p.slots[t] : -1;
    return s < slots_all ? s : -1;
  };
  const int mine = lane < chunk ? slot_of(t0 + lane) : -1, prev = slot_of(t0 + lane - 1);
  unsigned long long owners = __ballot(mine >= 0 && ((mine & (page - 1)) == 0 || prev != mine - 1));
  const int col = (lane % COLS) * 8, r0 = lane / COLS;
  while (owners) {
    const int own = __builtin_ctzll(owners);
    owners &= owners - 1;
    const long long t = t0 + own;
    const int s0 = __builtin_amdgcn_readlane(mine, own), o0 = s0 & (page - 1);
    const long long at = static_cast<long long>(s0 >> lp) * p.H + h, base = (at << lp) * D + col;
    const Incoming<T, F, D, MOVE> incoming(p, h, col);
    // New row i is row o0 + i of the page.
    CacheEight<T, F, D> k[U], v[U];
    const long long left = min(p.tokens - t, static_cast<long long>(page - o0));
    auto fetch = [&](int first) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = first + ROWS * u + r0;
        if (i < left) incoming.fetch(t + i, k[u], v[u]);
      }
    };
    fetch(0);
    int n = page - o0;  // end of the run of consecutive slots within the page
    for (int i = 0; i < n; i += 64) {
      const unsigned long long missing = __ballot(slot_of(t + i + lane) != s0 + i + lane);
      if (missing) n = min(n, i + static_cast<int>(__builtin_ctzll(missing)));
    }
    Extremes<T> seen;
    for (int first = 0; first < n; first += ROWS * U) {
      if (first > 0) fetch(first);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = first + ROWS * u + r0;
        if (i >= n) continue;
        write_row<MOVE>(p, base + (o0 + i) * D, k[u], v[u]);
        add_to(seen, k[u]);
      }
    }
    for (int first = r0; first < o0; first += ROWS * U) {  // older rows
      CacheEight<T, F, D> old[U];
#pragma unroll
      for (int u = 0; u < U; ++u) old[u].load(p.k_pages, base + min(first + ROWS * u, o0 - 1) * D);  // some of them twice
#pragma unroll
      for (int u = 0; u < U; ++u) add_to(seen, old[u]);
    }
    const int rows = o0 + n;
    float top[8], low[8];
    if (__any(seen.finish(top, low))) {
      __threadfence_block();  // rows that other lanes have written
      fold_with_nan<T, F, D>(p.k_pages, base, r0, ROWS, rows, top, low);
    }
    fold_rows<COLS>(top, low);
    store_bounds<D>(p, at, lane, top, low);
  }
}

template <class T, Format F, bool MOVE>
hipError_t launch(const PagedAppendArgs& a, hipStream_t stream) {
  const long long units = a.tokens * a.H;  // pages that the call can touch, times heads
  auto run = [&](auto d) {
    constexpr int D = decltype(d)::value;
    auto grid = [&](int pieces) { return dim3(static_cast<unsigned>((units * pieces + LANES - 1) / LANES)); };
    if (!a.bounds && MOVE) {
      const int bytes = F == E2M1 ? D / 2 : paged::row_bytes<T, F>(D);
      hipLaunchKernelGGL((paged_move_kernel<T, F, D>), grid(bytes / 16), dim3(LANES), 0, stream, a);
    } else if (!a.bounds) {
      hipLaunchKernelGGL((paged_append_kernel<T, F, D>), grid(D / 8), dim3(LANES), 0, stream, a);
    } else if (units <= FEW_PAGES) {
      hipLaunchKernelGGL((paged_append_bounds_kernel<T, F, D, MOVE>), dim3(static_cast<unsigned>(units)), dim3(LANES), 0, stream, a);
    } else {
      // About one owner to a wavefront: one without costs its start, one with two takes twice the chain.  12 prompts, 12000
      // tokens, 8 heads, d = 128, 8-bit pages, chunks of 12, 24, 48: pages of 16 22.3, 22.6, 25.8 us, of 32 25.1, 21.0, 23.7, of 64
      // 24.8, 21.4, 25.2 (22.8 with the 46 that they get here).
      const int chunk = static_cast<int>(std::min<long long>(std::max<long long>(units / 2048, 1), std::min(64, 3 << a.page_log2 >> 2)));
      const long long groups = (a.tokens + chunk * (LANES / 64) - 1) / (chunk * (LANES / 64));
      hipLaunchKernelGGL((paged_append_pages_kernel<T, F, D, MOVE>), dim3(static_cast<unsigned>(groups * a.H)), dim3(LANES), 0, stream, a,
                         chunk);
    }
  };
  if (a.d == 128)
    run(std::integral_constant<int, 128>{});
  else
    run(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

template <bool MOVE>
hipError_t launch(const PagedAppendArgs& a, hipStream_t stream) {
  if (a.tokens == 0) return hipSuccess;
  if (a.dtype == HEATKV_F32) return launch<float, NATIVE, MOVE>(a, stream);
  return a.kv_format == HEATKV_KV_FP4_E2M1   ? launch<bf16_t, E2M1, MOVE>(a, stream)
         : a.kv_format == HEATKV_KV_FP8_E4M3 ? launch<bf16_t, E4M3, MOVE>(a, stream)
                                             : launch<bf16_t, NATIVE, MOVE>(a, stream);
}

// The other way: rows of the cache by their slots, as values of the operands' type.
template <class T, Format F, int D>
__global__ __launch_bounds__(LANES) void paged_read_kernel(PagedReadArgs p) {
  const RowPiece r = row_piece<D / 8>(p.H);
  if (r.t >= p.tokens) return;
  const int slot = p.slots[r.t];
  if (!in_cache(p, slot)) return;
  const long long at = cache_row(p, slot, r.h) * D + 8 * r.piece;
  CacheEight<T, F, D> k, v;
  k.load(p.k_pages, at);
  v.load(p.v_pages, at);
  uint4 x[sizeof(T) / 2], y[sizeof(T) / 2];
  k.decode(x);
  v.decode(y);
  T* ko = static_cast<T*>(p.k_out) + r.t * p.k_token_stride + r.h * p.k_head_stride + 8 * r.piece;
  T* vo = static_cast<T*>(p.v_out) + r.t * p.v_token_stride + r.h * p.v_head_stride + 8 * r.piece;
#pragma unroll
  for (int j = 0; j < static_cast<int>(sizeof(T)) / 2; ++j) {
    *reinterpret_cast<uint4*>(ko + 4 * j) = x[j];
    *reinterpret_cast<uint4*>(vo + 4 * j) = y[j];
  }
}

template <class T, Format F>
hipError_t launch_read(const PagedReadArgs& a, hipStream_t stream) {
  const long long lanes = a.tokens * a.H * (a.d / 8);
  const dim3 grid(static_cast<unsigned>((lanes + LANES - 1) / LANES));
  if (a.d == 128)
    hipLaunchKernelGGL((paged_read_kernel<T, F, 128>), grid, dim3(LANES), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_read_kernel<T, F, 64>), grid, dim3(LANES), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream) {
  return a.from ? launch<true>(a, stream) : launch<false>(a, stream);
}

hipError_t launch_paged_read(const PagedReadArgs& a, hipStream_t stream) {
  if (a.tokens == 0) return hipSuccess;
  if (a.dtype == HEATKV_F32) return launch_read<float, NATIVE>(a, stream);
  return a.kv_format == HEATKV_KV_FP4_E2M1   ? launch_read<bf16_t, E2M1>(a, stream)
         : a.kv_format == HEATKV_KV_FP8_E4M3 ? launch_read<bf16_t, E4M3>(a, stream)
                                             : launch_read<bf16_t, NATIVE>(a, stream);
}

}  // namespace heatkv
