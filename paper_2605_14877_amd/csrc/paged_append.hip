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
// running state that would have to follow when tokens are dropped or pages change owners.
#include "copy_rows.h"
#include "kernels.h"
#include "paged.h"

namespace heatkv {

namespace {

constexpr int LANES = 256;

// 8 values of a row, as floats.
struct Eight {
  float v[8];
};
template <class T>
__device__ __forceinline__ void load8(const T* p, Eight& x, uint4 (&raw)[2]) {
  raw[0] = ldg16(p);
  if constexpr (sizeof(T) == 4) {
    raw[1] = ldg16(p + 4);
    const unsigned w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = __uint_as_float(w[i]);
  } else {
    const unsigned w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.v[2 * i] = __uint_as_float(w[i] << 16);
      x.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void decode8(uint2 w, Eight& x) {  // E4M3 codes
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = static_cast<int>(i ? w.y : w.x);
    x.v[4 * i] = __builtin_amdgcn_cvt_f32_fp8(c, 0);
    x.v[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8(c, 1);
    x.v[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8(c, 2);
    x.v[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8(c, 3);
  }
}

// Rows only: 8 elements of K and of V per lane.
template <class T, bool FP8>
__global__ __launch_bounds__(LANES) void paged_append_kernel(PagedAppendArgs p) {
  const int cpr = p.d / 8;
  const long long i = static_cast<long long>(blockIdx.x) * LANES + threadIdx.x;
  const int c = static_cast<int>(i & (cpr - 1));
  const long long row = p.d == 128 ? i >> 4 : i >> 3;
  const long long t = row / p.H;
  const int h = static_cast<int>(row - t * p.H);
  if (t >= p.tokens) return;
  const int slot = p.slots[t];
  if (slot < 0 || slot >= p.num_pages << p.page_log2) return;
  const T* k = static_cast<const T*>(p.k_new) + t * p.k_token_stride + h * p.k_head_stride + 8 * c;
  const T* v = static_cast<const T*>(p.v_new) + t * p.v_token_stride + h * p.v_head_stride + 8 * c;
  const long long to = ((((static_cast<long long>(slot >> p.page_log2) * p.H + h) << p.page_log2) +
                         (slot & ((1 << p.page_log2) - 1))) * p.d + 8 * c);
  if constexpr (FP8) {
    const uint4 a = ldg16(k), b = ldg16(v);
    *reinterpret_cast<uint2*>(static_cast<char*>(p.k_pages) + to) = make_uint2(bf16x4_to_e4m3(a.x, a.y), bf16x4_to_e4m3(a.z, a.w));
    *reinterpret_cast<uint2*>(static_cast<char*>(p.v_pages) + to) = make_uint2(bf16x4_to_e4m3(b.x, b.y), bf16x4_to_e4m3(b.z, b.w));
  } else {
    uint4* kd = reinterpret_cast<uint4*>(static_cast<T*>(p.k_pages) + to);
    uint4* vd = reinterpret_cast<uint4*>(static_cast<T*>(p.v_pages) + to);
    constexpr int N = sizeof(T) / 2;
    uint4 a[N], b[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      a[j] = ldg16(k + 4 * j);
      b[j] = ldg16(v + 4 * j);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      kd[j] = a[j];
      vd[j] = b[j];
    }
  }
}

// With bounds.  The first token of a call on a page is that page's owner: its workgroup writes all rows that the call
// brings to the page (tokens of one page follow one another, as the allocator hands out slots) and reads the rows that
// were there before.  A workgroup looks at `chunk` tokens (at most 64) of one kv head.
template <class T, bool FP8, int D>
__global__ __launch_bounds__(LANES) void paged_append_bounds_kernel(PagedAppendArgs p, int chunk) {
  constexpr int COLS = D / 8, ROWS = LANES / COLS;  // lanes of a row, rows side by side
  __shared__ float part[LANES / 64][2][D];
  __shared__ int run_end[LANES / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.y, lp = p.page_log2, page = 1 << lp;
  const long long t0 = static_cast<long long>(blockIdx.x) * chunk;
  const int slots_all = p.num_pages << lp;
  auto slot_of = [&](long long t) {
    const int s = t >= 0 && t < p.tokens ? p.slots[t] : -1;
    return s < slots_all ? s : -1;
  };
  unsigned long long owners;
  {
    const long long t = t0 + lane;
    const int s = lane < chunk ? slot_of(t) : -1, prev = slot_of(t - 1);
    owners = __ballot(s >= 0 && ((s & (page - 1)) == 0 || prev != s - 1));
  }
  const int col = (tid % COLS) * 8, r0 = tid / COLS;
  while (owners) {  // the same in all wavefronts
    const int own = __builtin_ctzll(owners);
    owners &= owners - 1;
    const long long t = t0 + own;
    const int s0 = p.slots[t], o0 = s0 & (page - 1);
    // end of the run of consecutive slots, within the page: `page` is at most the number of lanes
    const bool in_run = tid < page - o0 && slot_of(t + tid) == s0 + tid;
    const unsigned long long missing = __ballot(!in_run);
    if (lane == 0) run_end[wave] = missing ? 64 * wave + __builtin_ctzll(missing) : 1 << 30;
    __syncthreads();
    int n = run_end[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) n = min(n, run_end[w]);
    n = min(n, page - o0);
    const long long base = ((static_cast<long long>(s0 >> lp) * p.H + h) << lp) * D;
    const T* k_new = static_cast<const T*>(p.k_new) + h * p.k_head_stride + col;
    const T* v_new = static_cast<const T*>(p.v_new) + h * p.v_head_stride + col;
    float top[8], low[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = low[i] = -INFINITY;
    for (int r = r0; r < o0 + n; r += ROWS) {
      Eight x;
      uint4 raw[2];
      const long long at = base + static_cast<long long>(r) * D + col;
      if (r >= o0) {
        const long long tr = t + r - o0;
        load8(k_new + tr * p.k_token_stride, x, raw);
        const T* v = v_new + tr * p.v_token_stride;
        if constexpr (FP8) {
          const uint2 codes = make_uint2(bf16x4_to_e4m3(raw[0].x, raw[0].y), bf16x4_to_e4m3(raw[0].z, raw[0].w));
          const uint4 b = ldg16(v);
          *reinterpret_cast<uint2*>(static_cast<char*>(p.k_pages) + at) = codes;
          *reinterpret_cast<uint2*>(static_cast<char*>(p.v_pages) + at) =
              make_uint2(bf16x4_to_e4m3(b.x, b.y), bf16x4_to_e4m3(b.z, b.w));
          decode8(codes, x);
        } else {
#pragma unroll
          for (int j = 0; j < static_cast<int>(sizeof(T)) / 2; ++j) {
            const uint4 b = ldg16(v + 4 * j);
            *reinterpret_cast<uint4*>(static_cast<T*>(p.k_pages) + at + 4 * j) = raw[j];
            *reinterpret_cast<uint4*>(static_cast<T*>(p.v_pages) + at + 4 * j) = b;
          }
        }
      } else if constexpr (FP8) {
        decode8(*reinterpret_cast<const uint2*>(static_cast<const char*>(p.k_pages) + at), x);
      } else {
        load8(static_cast<const T*>(p.k_pages) + at, x, raw);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = x.v[i] == x.v[i] ? fminf(fmaxf(x.v[i], -0x1p127f), 0x1p127f) : 0.f;
        top[i] = fmaxf(top[i], y);
        low[i] = fmaxf(low[i], -y);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int m = COLS; m < 64; m *= 2) {
        top[i] = fmaxf(top[i], __shfl_xor(top[i], m, 64));
        low[i] = fmaxf(low[i], __shfl_xor(low[i], m, 64));
      }
    if (lane < COLS)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        part[wave][0][col + i] = top[i];
        part[wave][1][col + i] = low[i];
      }
    __syncthreads();
    if (wave == 0) {  // 2 D values, D / 32 per lane; a lane's lie side by side
      constexpr int N = 2 * D / 64;
      float x[N], amax = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float* q = &part[0][0][0] + lane * N + i;
        x[i] = q[0];
#pragma unroll
        for (int w = 1; w < LANES / 64; ++w) x[i] = fmaxf(x[i], q[w * 2 * D]);
        amax = fmaxf(amax, fabsf(x[i]));
      }
#pragma unroll
      for (int m = 1; m < 64; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
      const int e = paged::code_exponent(amax);
      union {
        int8_t c[N];
        unsigned short h[N / 2];
      } u;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int8_t code = static_cast<int8_t>(ceilf(ldexpf(x[i], -e)));
        u.c[i] = code == 0 && x[i] > 0.f ? 1 : code;  // upwards also where the quotient underflows
      }
      const long long at = (static_cast<long long>(s0 >> lp) * p.H + h);
      unsigned short* codes = reinterpret_cast<unsigned short*>(p.bounds + at * (2 * D)) + lane * (N / 2);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) codes[i] = u.h[i];
      if (lane == 0) p.bound_scales[at] = ldexpf(1.f, e);
    }
    __syncthreads();  // part and run_end are free again
  }
}

template <class T, bool FP8>
hipError_t launch(const PagedAppendArgs& a, hipStream_t stream) {
  if (!a.bounds) {
    const long long lanes = a.tokens * a.H * (a.d / 8);
    hipLaunchKernelGGL((paged_append_kernel<T, FP8>), dim3(static_cast<unsigned>((lanes + LANES - 1) / LANES)), dim3(LANES), 0,
                       stream, a);
    return hipGetLastError();
  }
  // A workgroup per token and head while that fills the chip (single tokens: every one owns a page), up to 64 tokens, more
  // than one page of the smallest size, beyond.
  const int chunk = static_cast<int>(std::min<long long>(std::max<long long>(a.tokens * a.H / 4096, 1), 64));
  const dim3 grid(static_cast<unsigned>((a.tokens + chunk - 1) / chunk), a.H);
  if (a.d == 128)
    hipLaunchKernelGGL((paged_append_bounds_kernel<T, FP8, 128>), grid, dim3(LANES), 0, stream, a, chunk);
  else
    hipLaunchKernelGGL((paged_append_bounds_kernel<T, FP8, 64>), grid, dim3(LANES), 0, stream, a, chunk);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream) {
  if (a.tokens == 0) return hipSuccess;
  if (a.dtype == HEATKV_F32) return launch<float, false>(a, stream);
  return a.kv_fp8 ? launch<bf16_t, true>(a, stream) : launch<bf16_t, false>(a, stream);
}

}  // namespace heatkv
