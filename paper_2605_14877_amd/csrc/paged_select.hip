// Paged cache: the pages that each new token's attention reads, chosen by a score over the pages' 8-bit bounds.
//
// score(page) = sum over the queries of the kv head's group of the largest value that q . k takes for any key within the
// page's bounds = sum_d (a_d top_d + b_d low_d), where a and b are the group's sums of the positive and of the negated
// negative parts of its queries, top and low the largest and minus the smallest key value (paged_append.hip).  Queries are
// rounded to 8-bit codes with one power of two per token and group, which leaves the order of the pages alone, so a score
// is a dot product of whole numbers of 2 d terms, times the page's own power of two: the matrix cores form it exactly in
// int32 (a and b, up to 16 x 127, as two 7-bit digits), and it is rounded once, to fp32.  A choice is therefore
// reproducible bit for bit, however the work is cut; equal scores go to the lower page.
//
// A workgroup takes TW tokens of a request and a kv head, scores all pages that the last of them sees into LDS (16 pages a
// time and wavefront) and then ranks them token by token: the score of the last page to take is found by halving the
// interval of the scores, and a pass in page order writes what lies above it.
//
// Bound: latency, not the bytes of the bounds (2 d + 4 a page and head).  16 requests of up to 512 pages, 8 heads, d = 128: 14.6 to
// 16 us, without the ranking 10.9 (request, queries, codes, table and bounds one after another); 1024 tokens over 272 pages, 4
// heads: 21 us, without the ranking 12.
#include <hip/hip_runtime.h>

#include "attend_params.h"
#include "kernels.h"
#include "paged.h"
#include "paged_walk.h"

namespace heatkv {

namespace {

using namespace paged;

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int LANES = 256, WAVES = 4;
extern __shared__ __attribute__((aligned(16))) char select_lds[];

// Scores as unsigned numbers of the same order.  0: a page that the token does not see; FORCED: one that it takes anyway.
constexpr unsigned FORCED = 0xffffffffu;
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The bar that `top` scores reach: those above it are taken, of those equal to it as many as are missing then, from the lowest
// page on.  At least `top` scores are >= low, fewer are > high; count(x): how many are >= x.
template <class Count>
__device__ __forceinline__ unsigned bar_between(unsigned low, unsigned high, int top, const Count& count) {
  while (low < high) {
    const unsigned mid = low + (high - low + 1) / 2;
    const int c = count(mid);
    if (c == top) return mid - 1;  // exactly these
    if (c > top)
      low = mid;
    else
      high = mid - 1;
  }
  return low;
}

template <int TW, int D>
constexpr int digit_bytes() { return TW * 2 * 2 * D; }

// N consecutive query values (8 or 4, a multiple of 8 bytes).
template <class T, int N>
__device__ __forceinline__ void query_values(const T* p, float (&x)[N]) {
  typedef T Pack __attribute__((ext_vector_type(N)));
  const Pack y = *reinterpret_cast<const Pack*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float z = static_cast<float>(y[i]);
    x[i] = z == z ? fminf(fmaxf(z, -0x1p127f), 0x1p127f) : 0.f;
  }
}

// Ranks one token by one wavefront: up to 64 R scores, which stay in registers.
template <int R>
__device__ __forceinline__ void rank_token(const unsigned* key, int scan, int seen, int forced, int top, int* out, int lane) {
  unsigned k[R];
#pragma unroll
  for (int r = 0; r < R; ++r) k[r] = 64 * r + lane < scan ? key[64 * r + lane] : 0;
  auto count = [&](unsigned least) {
    int c = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) c += __popcll(__ballot(k[r] >= least));
    return c;
  };
  unsigned bar = 0;
  if (seen > top) {
    if (forced >= top) {
      bar = FORCED - 1;
    } else {
      unsigned low = FORCED, high = 0;
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (k[r] != 0 && k[r] != FORCED) {
          low = min(low, k[r]);
          high = max(high, k[r]);
        }
#pragma unroll
      for (int m = 1; m < 64; m *= 2) {
        low = min(low, static_cast<unsigned>(__shfl_xor(static_cast<int>(low), m, 64)));
        high = max(high, static_cast<unsigned>(__shfl_xor(static_cast<int>(high), m, 64)));
      }
      low = __builtin_amdgcn_readfirstlane(low);
      high = __builtin_amdgcn_readfirstlane(high);
      bar = bar_between(low, high, top, count);
    }
  }
  int ties = bar == 0 ? 0 : top - count(bar + 1), n = 0;
  const unsigned long long before = (1ull << lane) - 1;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const unsigned long long equal = __ballot(k[r] == bar);
    const bool take = k[r] > bar || (k[r] == bar && __popcll(equal & before) < ties);
    const unsigned long long taken = __ballot(take);
    if (take) out[n + __popcll(taken & before)] = 64 * r + lane;
    n += __popcll(taken);
    ties -= min(ties, static_cast<int>(__popcll(equal)));
  }
  for (int i = n + lane; i < top; i += 64) out[i] = -1;
}

// WPT wavefronts rank a token.
template <class T, int D, int TW, int WPT>
__global__ __launch_bounds__(LANES) void paged_select_kernel(PagedSelectParams p) {
  constexpr int KS = 2 * D / 64;  // MFMA steps of a score
  constexpr int COLS = D / 16;    // query columns of a lane
  constexpr int PARTS = LANES / 16 / TW;  // sets of 16 lanes that share a token's queries
  __shared__ unsigned amax_bits[TW];
  __shared__ unsigned counts[2][WAVES];
  signed char* const digits = reinterpret_cast<signed char*>(select_lds);  // [TW][2][2 D]
  int* const sums = reinterpret_cast<int*>(select_lds + digit_bytes<TW, D>());  // [TW][2 D], before the scores
  unsigned* const keys = reinterpret_cast<unsigned*>(sums);                     // [TW][pitch]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % p.c.H, pitch = p.pitch;
  const Tile tile = find_tile<TW>(p.tokens_as_rows, blockIdx.x / p.c.H, lane);
  if (tile.rows <= 0) return;
  const int page = 1 << p.c.page_log2;
  auto pages_seen = [&](int token) { return (visible_keys(p.c, tile, tile.row0 + token) + page - 1) >> p.c.page_log2; };

  // Query codes.
  for (int i = tid; i < TW * 2 * D; i += LANES) sums[i] = 0;
  if (tid < TW) amax_bits[tid] = 0;
  __syncthreads();
  {
    const int token = tid / (16 * PARTS), part = tid / 16 % PARTS, col = tid % 16 * COLS;
    const bool real = token < tile.rows;
    const T* q = static_cast<const T*>(p.q.data) + (tile.q0 + tile.row0 + (real ? token : 0)) * p.q.token_stride +
                 static_cast<long long>(h) * p.c.G * p.q.head_stride + col;
    float amax = 0.f, x[COLS];
    if (real)
      for (int g = part; g < p.c.G; g += PARTS) {
        query_values(q + g * p.q.head_stride, x);
#pragma unroll
        for (int i = 0; i < COLS; ++i) amax = fmaxf(amax, fabsf(x[i]));
      }
#pragma unroll
    for (int m = 1; m < 16; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
    if (tid % 16 == 0) atomicMax(&amax_bits[token], __float_as_uint(amax));  // not negative: ordered as their bits
    __syncthreads();
    const int e = code_exponent(__uint_as_float(amax_bits[token]));
    int up[COLS], down[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) up[i] = down[i] = 0;
    if (real)
      for (int g = part; g < p.c.G; g += PARTS) {
        query_values(q + g * p.q.head_stride, x);
#pragma unroll
        for (int i = 0; i < COLS; ++i) {
          const int code = static_cast<int>(rintf(ldexpf(x[i], -e)));
          up[i] += max(code, 0);
          down[i] += max(-code, 0);
        }
      }
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
      atomicAdd(&sums[token * 2 * D + col + i], up[i]);
      atomicAdd(&sums[token * 2 * D + D + col + i], down[i]);
    }
  }
  __syncthreads();
  for (int i = tid; i < TW * 2 * D; i += LANES) {
    const int token = i / (2 * D), k = i % (2 * D), v = sums[i];
    digits[(2 * token) * 2 * D + k] = static_cast<signed char>(v & 127);
    digits[(2 * token + 1) * 2 * D + k] = static_cast<signed char>(v >> 7);
  }
  __syncthreads();

  // Scores.  A: 16 pages, B: the tokens; lane (n, g) supplies 16 bytes of page / token n and holds pages 4 g + r, token n.
  const int n = lane & 15, g = lane >> 4;
  const int pages_all = pages_seen(tile.rows - 1);
  {
    i32x4 lo[KS], hi[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const i32x4 zero = {0, 0, 0, 0};
      const i32x4* b = reinterpret_cast<const i32x4*>(digits + 2 * (n < TW ? n : 0) * 2 * D + 64 * ks + 16 * g);
      lo[ks] = n < TW ? b[0] : zero;
      hi[ks] = n < TW ? b[2 * D / 16] : zero;
    }
    const int* table = p.c.table + static_cast<long long>(tile.b) * p.c.max_pages;
    const int seen = n < tile.rows ? pages_seen(n) : 0;
    constexpr int U = 4;  // groups of 16 pages whose loads are under way together
    for (int g0 = wave; g0 * 16 < pages_all; g0 += WAVES * U) {
      long long row[U];
      i32x4 a[U][KS];
      float scale[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = min((g0 + u * WAVES) * 16 + n, p.c.max_pages - 1);
        row[u] = static_cast<long long>(min(static_cast<unsigned>(table[x]), static_cast<unsigned>(p.c.num_pages - 1))) * p.c.H + h;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const i32x4* from = reinterpret_cast<const i32x4*>(p.bounds + row[u] * (2 * D) + 16 * g);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) a[u][ks] = from[4 * ks];
        scale[u] = p.bound_scales[row[u]];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int first = (g0 + u * WAVES) * 16;
        if (first >= pages_all) break;
        i32x4 s = {0, 0, 0, 0}, t = {0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][ks], lo[ks], s, 0, 0, 0);
        if (p.c.G > 1)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) t = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][ks], hi[ks], t, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = first + 4 * g + r;
          const float score = static_cast<float>(s[r] + (t[r] << 7)) * __shfl(scale[u], 4 * g + r, 64);
          unsigned key = x < seen ? min(max(ordered(score), 1u), FORCED - 1) : 0u;
          if (x < seen && (x < p.first || x >= seen - p.last)) key = FORCED;
          if (n < TW) keys[n * pitch + x] = key;
        }
      }
    }
  }
  __syncthreads();

  // Ranking: a wavefront per token where the scores fit into its registers.
  const int scan = (pages_all + 15) / 16 * 16;
  auto output = [&](int token) {
    return p.selected + (static_cast<long long>(tile.q0 + tile.row0 + token) * p.c.H + h) * p.top;
  };
  auto forced_of = [&](int seen) { return min(seen, p.first) + max(0, min(p.last, seen - p.first)); };
  if (scan <= 1024) {
    for (int token = wave; token < tile.rows; token += WAVES) {
      const unsigned* key = keys + token * pitch;
      const int seen = pages_seen(token), forced = forced_of(seen);
      if (scan <= 128)
        rank_token<2>(key, scan, seen, forced, p.top, output(token), lane);
      else if (scan <= 320)
        rank_token<5>(key, scan, seen, forced, p.top, output(token), lane);
      else if (scan <= 512)
        rank_token<8>(key, scan, seen, forced, p.top, output(token), lane);
      else
        rank_token<16>(key, scan, seen, forced, p.top, output(token), lane);
    }
    return;
  }
  for (int token = wave / WPT; token < tile.rows; token += WAVES / WPT) {
    const unsigned* key = keys + token * pitch;
    const int seen = pages_seen(token), forced = forced_of(seen);
    // Sum of a count over the lanes that rank this token; the same number on all of them.
    int turn = 0;
    auto total = [&](unsigned c) {
      c = __builtin_amdgcn_readfirstlane(c);
      if constexpr (WPT > 1) {
        if (lane == 0) counts[turn][wave] = c;
        __syncthreads();
        c = counts[turn][0] + counts[turn][1] + counts[turn][2] + counts[turn][3];
        turn ^= 1;  // the next round's counts are written while others may still read these
      }
      return static_cast<int>(c);
    };
    const int sub = WPT > 1 ? tid : lane, stride = 64 * WPT;
    auto count_from = [&](unsigned least) {
      unsigned c = 0;
      for (int i = sub; i - lane < scan; i += stride) c += __popcll(__ballot(i < scan && key[i] >= least));
      return total(c);
    };
    unsigned bar = 0;
    if (seen > p.top) {
      if (forced >= p.top) {
        bar = FORCED - 1;
      } else {
        unsigned low = FORCED, high = 0;
        for (int i = sub; i < scan; i += stride) {
          const unsigned k = key[i];
          if (k != 0 && k != FORCED) {
            low = min(low, k);
            high = max(high, k);
          }
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
          low = min(low, static_cast<unsigned>(__shfl_xor(static_cast<int>(low), m, 64)));
          high = max(high, static_cast<unsigned>(__shfl_xor(static_cast<int>(high), m, 64)));
        }
        if constexpr (WPT > 1) {
          if (lane == 0) {
            counts[0][wave] = low;
            counts[1][wave] = high;
          }
          __syncthreads();
#pragma unroll
          for (int w = 0; w < WAVES; ++w) {
            low = min(low, counts[0][w]);
            high = max(high, counts[1][w]);
          }
          __syncthreads();
        }
        bar = bar_between(low, high, p.top, count_from);
      }
    }
    // In page order, by one wavefront.
    if (WPT > 1 && wave > 0) continue;
    int above = 0;
    for (int i = lane; i - lane < scan; i += 64) above += __popcll(__ballot(i < scan && key[i] > bar));
    int ties = bar == 0 ? 0 : p.top - above, n = 0;
    int* const out = output(token);
    const unsigned long long before = (1ull << lane) - 1;
    for (int i = lane; i - lane < scan; i += 64) {
      const unsigned k = i < scan ? key[i] : 0;
      const unsigned long long equal = __ballot(i < scan && k == bar);
      const bool take = i < scan && (k > bar || (k == bar && __popcll(equal & before) < ties));
      const unsigned long long taken = __ballot(take);
      if (take) out[n + __popcll(taken & before)] = i;
      n += __popcll(taken);
      ties -= min(ties, static_cast<int>(__popcll(equal)));
    }
    for (int i = n + lane; i < p.top; i += 64) out[i] = -1;
  }
}

template <class T, int D, int TW, int WPT>
hipError_t launch(const PagedSelectParams& p, size_t lds, hipStream_t stream) {
  static std::atomic<unsigned long long> allowed{0};
  if (lds > 64 * 1024)
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(&paged_select_kernel<T, D, TW, WPT>), PAGED_SELECT_LDS, allowed))
      return e;
  const unsigned tiles = static_cast<unsigned>(tile_count<TW>(p.c.tokens, 1, p.c.batch));
  hipLaunchKernelGGL((paged_select_kernel<T, D, TW, WPT>), dim3(tiles * p.c.H), dim3(LANES), lds, stream, p);
  return hipGetLastError();
}

template <class T, int D>
hipError_t launch(PagedSelectParams p, hipStream_t stream) {
  p.pitch = (p.c.max_pages + 15) / 16 * 16;
  auto lds = [&](int tw) { return static_cast<size_t>(tw) * (4 * D + 4 * static_cast<size_t>(std::max(p.pitch, 2 * D))); };
  // Tokens of a request share a pass over the bounds: one, four or sixteen to a workgroup, as many as leave work for half of the
  // compute units with four, for all of them, four workgroups each, with sixteen, and whose scores fit into the LDS.  4 kv heads
  // over 272 pages, 16, 4 and 1 tokens to a workgroup: 64 new tokens 19.1, 10.7, 9.9 us, 128 18.8, 10.5, 11.8, 768 19.9, 15.9,
  // 44.2, 1024 19.8, 23.9, 57.4.  Little more than one token for each request: one.
  const long long units = static_cast<long long>(p.c.tokens) * p.c.H;
  if (p.c.tokens > 2 * p.c.batch + 16) {
    if (units >= 4 * 1024 && lds(16) <= 80 * 1024) return launch<T, D, 16, 1>(p, lds(16), stream);
    if (units >= 512 && lds(4) <= PAGED_SELECT_LDS) return launch<T, D, 4, 1>(p, lds(4), stream);
  }
  return launch<T, D, 1, WAVES>(p, lds(1), stream);
}

}  // namespace

hipError_t launch_paged_select(const PagedSelectParams& p, int dtype, int d, hipStream_t stream) {
  if (p.c.tokens == 0) return hipSuccess;
  if (dtype == HEATKV_F32) return d == 128 ? launch<float, 128>(p, stream) : launch<float, 64>(p, stream);
  return d == 128 ? launch<bf16_t, 128>(p, stream) : launch<bf16_t, 64>(p, stream);
}

}  // namespace heatkv
