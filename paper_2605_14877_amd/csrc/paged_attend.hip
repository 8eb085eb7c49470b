// Attention of new tokens over the paged cache, bf16 (cache rows bf16 or FP8 E4M3): few query rows per request, or a choice
// of pages for each token.  paged_attend_long.hip: many rows over all pages; paged_attend_f32.hip: fp32.
//
// A workgroup takes its share of the launch (paged_schedule.h), segment by segment: 16 query rows (tokens x the queries that
// share a kv head) and a range of their keys.  Its four wavefronts take the range's steps of 32 keys in turn, each with a
// running reference, row sums and accumulators of its own, merged through LDS at the end of the segment.
//
// S^T = K Q^T with v_mfma_f32_16x16x32_bf16: K rows come from memory straight into the A operand (16 bytes per lane; the
// elements of a row may be dealt to the MFMA steps in any order that Q follows, so 8-bit rows are read 16 codes a lane as
// well).  Lane (n, g) then holds keys 4 g .. 4 g + 3 of two granules for query n, which is the B operand of
// O^T += V^T P^T as it stands if V's rows are taken in that order.  V^T is the A operand, out of a wavefront-private LDS
// stage by the transposing read; windows of 32 bytes of a row are XORed with the row number so that the eight rows of a
// read lie on different banks.
//
// Bound: HBM (K and V are read once for 16 rows): 64 requests of 4500 keys on average, 32 heads over 8, d = 128: 1.19 GB in 206
// us, 5.8 TB/s.  Small launches: the first loads and the merge, one 8-bit request of 65536 keys 134 MB in 30 us, 32 chosen pages
// of 64 keys for each of 16 requests and 8 heads as much in as long.
#include <hip/hip_runtime.h>

#include "f32_mfma.h"
#include "kernels.h"
#include "paged.h"
#include "paged_redo.h"
#include "paged_schedule.h"
#include "paged_walk.h"

namespace heatkv {

namespace {

using namespace paged;

constexpr int WAVES = 4, STEP = 32;  // wavefronts of a workgroup, keys of a step
extern __shared__ __attribute__((aligned(16))) char paged_lds[];

// 8 or 16 E4M3 codes as bf16 (exact).
__device__ __forceinline__ bf16x8 codes_to_bf16(unsigned lo, unsigned hi) {
  union {
    bf16x2 h[4];
    bf16x8 v;
  } o;
  o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(lo), 1.0f, false);
  o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(lo), 1.0f, true);
  o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(hi), 1.0f, false);
  o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(hi), 1.0f, true);
  return o.v;
}

template <int D, bool FP8, bool CHOSEN>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_attend_kernel(AttendParams p) {
  constexpr int NK = D / 32, NV = D / 16;            // MFMA steps of a score, accumulator blocks of 16 columns
  constexpr int RB = 2 * D;                          // bytes of a bf16 row in the V stage
  constexpr int SRC = FP8 ? D : 2 * D;               // bytes of a cache row
  constexpr int KC = SRC / 64, VC = STEP * SRC / 1024;  // 16-byte loads per lane: a granule of K, a step of V
  constexpr int LPR = SRC / 16;                      // lanes that share a row of V
  constexpr int RPL = 64 / LPR;                      // rows of V per load
  constexpr int PITCH = D + 4;                       // floats per row of a parked output tile
  static_assert(16 * PITCH * 4 == stage_bytes(D) && STEP * RB <= stage_bytes(D), "the parked tiles take the stages' place");
  char* const stage_all = paged_lds;                 // [WAVES] V stages, then the parked output tiles
  __shared__ float part_m[WAVES][16], part_l[WAVES][16];

  __shared__ Line line;
  __shared__ unsigned nan_rows;

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = blockIdx.x;
  line.start<16, STEP>(p, w);
  Part part;
  for (bool first = true; line.advance<16, STEP>(p, first, part); first = false) {
    const Tile tile = tile_of<16>(p.c, part);
    const int h = part.h;

    // This lane's query row.
    const int row = tile.row0 + min(n, tile.rows - 1);
    const int j = divide(row, p.c.div_G), hq = h * p.c.G + row - j * p.c.G;
    const long long token = tile.q0 + j;
    const int limit = n < tile.rows ? visible_keys(p.c, tile, j) : 0;
    const int j_last = divide(tile.row0 + tile.rows - 1, p.c.div_G), j_first = divide(tile.row0, p.c.div_G);
    const int limit_max = visible_keys(p.c, tile, j_last), limit_min = tile.rows == 16 ? visible_keys(p.c, tile, j_first) : 0;

    Walk<CHOSEN> walk(p, tile, h, j_first, j_last, limit_max, paged_lds + WAVES * stage_bytes(D), tid);
    const int steps = walk.steps();
    const int begin = steps_before(part.from, part.weight, steps), end = steps_before(part.to, part.weight, steps);

    bf16x8 q[NK];
    {
      const bf16_t* from = static_cast<const bf16_t*>(p.q.data) + token * p.q.token_stride + hq * p.q.head_stride;
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        const int at = FP8 ? 64 * (ks / 2) + 16 * g + 8 * (ks % 2) : 32 * ks + 8 * g;
        q[ks] = *reinterpret_cast<const bf16x8*>(from + at);
      }
    }
    const char* const k_pages = static_cast<const char*>(p.k_pages);
    const char* const v_pages = static_cast<const char*>(p.v_pages);
    const unsigned k_off = n * SRC + 16 * g;
    const unsigned v_off = (lane / LPR) * SRC + (lane % LPR) * 16;

    uint4 k_raw[2][KC], v_raw[VC];
    Granule at[2] = {};
    auto fetch_k = [&] {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < KC; ++c) k_raw[i][c] = ldg16(k_pages + at[i].row * SRC + k_off + 64 * c);
    };
    auto fetch_v = [&] {
#pragma unroll
      for (int c = 0; c < VC; ++c) v_raw[c] = ldg16(v_pages + at[c / (VC / 2)].row * SRC + v_off + (c % (VC / 2)) * 1024);
    };

    f32x4 o[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = p.sm_scale * kLog2e;
    float m = lowest_reference(c), l = 0.f;
    constexpr float kSlack = 8.f;  // the reference is raised by more than this only: attend.hip
    const float slack = kSlack / c;
    char* const stage = stage_all + wave * stage_bytes(D);
    // Reader of the stage: lane i of group g points at row 4 g + i / 4, column 4 (i % 4) of a block of 16.
    const int v_row = 4 * g + (n >> 2);

    int step = begin + wave;
    Granule next[2] = {};
    if (step < end) {
      at[0] = walk.locate(2 * step);
      at[1] = walk.locate(2 * step + 1);
      fetch_k();
      fetch_v();
    }
    while (step < end) {
      const int step_next = step + WAVES;
      const bool more = step_next < end;
      if (more) {
        next[0] = walk.locate(2 * step_next);
        next[1] = walk.locate(2 * step_next + 1);
      }
      // Scores of two granules, lane (n, g): keys 4 g + r.
      f32x4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
          bf16x8 a;
          if constexpr (FP8) {
            const uint4& w = k_raw[i][ks / 2];
            a = ks % 2 ? codes_to_bf16(w.z, w.w) : codes_to_bf16(w.x, w.y);
          } else {
            a = __builtin_bit_cast(bf16x8, k_raw[i][ks]);
          }
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[ks], s[i], 0, 0, 0);
        }
      }
      // V into the stage; rows behind the request's end as zeros (a probability of 0 does not remove an infinity).
#pragma unroll
      for (int cidx = 0; cidx < VC; ++cidx) {
        const int i = cidx / (VC / 2), r = (cidx % (VC / 2)) * RPL + lane / LPR;  // granule, row of it
        uint4 w = v_raw[cidx];
        if (at[i].pos + GRANULE > tile.len && at[i].pos + r >= tile.len) w = make_uint4(0, 0, 0, 0);
        const int row_in = 16 * i + r;
        if constexpr (FP8) {
          const int win = (lane % LPR) ^ stage_swizzle<D>(row_in);
          bf16x8* to = reinterpret_cast<bf16x8*>(stage + row_in * RB + win * 32);
          to[0] = codes_to_bf16(w.x, w.y);
          to[1] = codes_to_bf16(w.z, w.w);
        } else {
          const int chunk = lane % LPR, win = (chunk >> 1) ^ stage_swizzle<D>(row_in);
          *reinterpret_cast<uint4*>(stage + row_in * RB + win * 32 + (chunk & 1) * 16) = w;
        }
      }
      const Granule here[2] = {at[0], at[1]};
      if (more) {
        at[0] = next[0];
        at[1] = next[1];
        fetch_k();
        fetch_v();
      }
      // Keys that a row does not see.
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (here[i].pos + GRANULE > limit_min || CHOSEN) {
          const int lim = walk.sees(here[i], j - j_first) ? limit - here[i].pos - 4 * g : 0;
#pragma unroll
          for (int r = 0; r < 4; ++r) s[i][r] = r < lim ? s[i][r] : -INFINITY;
        }
      }
      const float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                             fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      if (__any(mx > m + slack)) {
        const float m_new = fmaxf(m, f32m::max_groups(mx));
        const float alpha = fast_exp2((m - m_new) * c);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < NV; ++i) o[i] *= alpha;
      }
      // Probabilities are rounded to bf16 for the product; the row sum takes them as they are (the logarithm of the sum is an
      // output, in fp32).
      bf16x8 pb;
      const float mc = m * c;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = fast_exp2(fmaf(s[i >> 2][i & 3], c, -mc));
        l += e;
        pb[i] = static_cast<bf16_t>(e);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        union {
          struct {
            s16x4 lo, hi;
          } s;
          bf16x8 v;
        } a;
        const char* from = stage + v_row * RB + ((i ^ stage_swizzle<D>(v_row)) * 32) + (n & 3) * 8;
        a.s.lo = lds_read_tr16(reinterpret_cast<const bf16_t*>(from));
        a.s.hi = lds_read_tr16(reinterpret_cast<const bf16_t*>(from + 16 * RB));
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pb, o[i], 0, 0, 0);
      }
      step = step_next;
    }

    // Merge of the four wavefronts: each brings its accumulators to the common reference; the parked tiles are added in
    // wavefront order.  A wavefront without a step has the lowest reference and factor 0.
    __syncthreads();  // every wavefront is done with its stage
    l = f32m::sum_groups(l);
    if (g == 0) {
      part_m[wave][n] = m;
      part_l[wave][n] = l;
    }
    if (tid == 0) nan_rows = 0;
    const Part done = line.stored();
    const bool alone = done.from == 0 && done.to == done.weight;  // no other workgroup has a part of this segment
    const long long part_base = line.part_rows<16>(w, done);
    __syncthreads();
    float m_all = part_m[0][n], l_all = 0.f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m_all = fmaxf(m_all, part_m[w][n]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) l_all += part_l[w][n] * fast_exp2((part_m[w][n] - m_all) * c);
    const float to_all = fast_exp2((m - m_all) * c);
    const float f = !alone ? to_all : l_all > 0.f ? to_all / l_all : l_all;  // nothing seen: zeros; NaN stays
    float* const park = reinterpret_cast<float*>(stage_all);
#pragma unroll
    for (int i = 0; i < NV; ++i) *reinterpret_cast<f32x4*>(park + (wave * 16 + n) * PITCH + 16 * i + 4 * g) = o[i] * f;
    if (tid < tile.rows) {  // wave 0, g == 0 or not: lane = row
      const int r = divide(tile.row0 + tid, p.c.div_G);
      const long long out_row = (tile.q0 + r) * static_cast<long long>(p.c.Hq) + h * p.c.G + tile.row0 + tid - r * p.c.G;
      float ml = part_m[0][tid], ll = 0.f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) ml = fmaxf(ml, part_m[w][tid]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) ll += part_l[w][tid] * fast_exp2((part_m[w][tid] - ml) * c);
      if (!alone) {
        float* to = p.parts.ml + (part_base + tid) * 2;
        to[0] = ml;
        to[1] = ll;
      } else if (p.lse) {
        p.lse[out_row] = natural_lse(ml, ll, p.sm_scale);
      }
    }
    __syncthreads();
    for (int e = tid; e < tile.rows * (D / 8); e += 64 * WAVES) {
      const int r = e / (D / 8), col = e % (D / 8) * 8;
      f32x4 x[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        x[k] = *reinterpret_cast<const f32x4*>(park + r * PITCH + col + 4 * k);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x[k] += *reinterpret_cast<const f32x4*>(park + (w * 16 + r) * PITCH + col + 4 * k);
      }
      const int jr = divide(tile.row0 + r, p.c.div_G), hr = h * p.c.G + tile.row0 + r - jr * p.c.G;
      bool nan = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) nan = nan || x[k >> 2][k & 3] != x[k >> 2][k & 3];
      if (nan) atomicOr(&nan_rows, 1u << r);
      if (!alone) {
        float* to = p.parts.o + (part_base + r) * D + col;
        *reinterpret_cast<f32x4*>(to) = x[0];
        *reinterpret_cast<f32x4*>(to + 4) = x[1];
      } else {
        bf16x8 y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = static_cast<bf16_t>(x[k >> 2][k & 3]);
        bf16_t* to = static_cast<bf16_t*>(const_cast<void*>(p.out.data)) + (tile.q0 + jr) * p.out.token_stride + hr * p.out.head_stride + col;
        *reinterpret_cast<bf16x8*>(to) = y;
      }
    }
    __syncthreads();  // outputs are written; LDS is free for the next segment
    for (unsigned rows = nan_rows; rows;) {  // paged_redo.h
      const int r = __builtin_ctz(rows);
      rows &= rows - 1;
      if (r % WAVES != wave) continue;
      const AttendParams& z = arguments();
      const int jr = divide(tile.row0 + r, z.c.div_G), hr = h * z.c.G + tile.row0 + r - jr * z.c.G;
      float m_row = part_m[0][r], l_row = 0.f;
      for (int i = 1; i < WAVES; ++i) m_row = fmaxf(m_row, part_m[i][r]);
      for (int i = 0; i < WAVES; ++i) l_row += part_l[i][r] * fast_exp2((part_m[i][r] - m_row) * c);
      const float norm = !alone ? 1.f : l_row > 0.f ? 1.f / l_row : l_row;
      float* const parts_row = z.parts.o + (part_base + r) * D;  // the part's, or not used
      bf16_t* const out_row = static_cast<bf16_t*>(const_cast<void*>(z.out.data)) + (tile.q0 + jr) * z.out.token_stride + hr * z.out.head_stride;
      redo_row<bf16_t, FP8, D, CHOSEN>(
          z, tile.q0 + jr, hr, visible_keys(z.c, tile, jr), tile.len, 2 * begin, 2 * end, false,
          [&](int gr) {
            const Granule at = walk.locate(gr);
            return RedoGranule{at.row, at.pos, walk.sees(at, jr - j_first)};
          },
          [&](float score) { return fast_exp2((score - m_row) * c); },
          [&](int col) { return alone ? static_cast<float>(out_row[col]) : parts_row[col]; },
          [&](int col, float x, float) {
            if (!alone)
              parts_row[col] = x;
            else
              out_row[col] = static_cast<bf16_t>(x * norm);
          });
    }
    if (CHOSEN) __syncthreads();  // the walk's tables are free as well
  }
}

template <int D, bool FP8, bool CHOSEN>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  const size_t lds = WAVES * stage_bytes(D) + (CHOSEN ? walk_lds_bytes(p) : 0);
  static std::atomic<unsigned long long> allowed{0};
  if (lds > 64 * 1024)
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(&paged_attend_kernel<D, FP8, CHOSEN>), WALK_LDS, allowed)) return e;
  hipLaunchKernelGGL((paged_attend_kernel<D, FP8, CHOSEN>), dim3(p.parts.grid), dim3(64 * WAVES), lds, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attend_bf16(const PagedAttendParams& p, int d, bool fp8, hipStream_t stream) {
  if (p.selected) {
    if (d == 128) return fp8 ? launch<128, true, true>(p, stream) : launch<128, false, true>(p, stream);
    return fp8 ? launch<64, true, true>(p, stream) : launch<64, false, true>(p, stream);
  }
  if (d == 128) return fp8 ? launch<128, true, false>(p, stream) : launch<128, false, false>(p, stream);
  return fp8 ? launch<64, true, false>(p, stream) : launch<64, false, false>(p, stream);
}

}  // namespace heatkv
