// Attention of new tokens over the paged cache, fp32 (paged_attend_few.h describes segments and walks; attend_f32.hip the
// operands and the arithmetic: K through a wavefront's LDS stage, V straight into registers, 16x16x4 fp32 MFMAs).
//
// A segment has 16 query rows; the workgroup's four wavefronts take granules of 16 keys in turn.
// Bound: HBM for single tokens; the fp32 matrix instructions and the vector work that does not overlap with them otherwise.
// Small launches: the chain of place, table, keys and merge, 11 us for 3 requests of 37 new tokens and up to 740 keys.
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

constexpr int WAVES = 4;
extern __shared__ __attribute__((aligned(1024))) char paged_f32_lds[];

template <int D, bool CHOSEN>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_attend_f32_kernel(AttendParams p) {
  constexpr int NB = D / 16, PITCH = D + 4;
  using Stage = f32m::KeyStage<D>;
  static_assert(16 * PITCH * 4 == stage_bytes(D) && Stage::BYTES <= stage_bytes(D), "the parked tiles take the stages' place");
  __shared__ float part_m[WAVES][16], part_l[WAVES][16];

  __shared__ Line line;
  __shared__ unsigned nan_rows;

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = blockIdx.x;
  line.start<16, 2 * GRANULE>(p, w);
  Part part;
  for (bool first = true; line.advance<16, 2 * GRANULE>(p, first, part); first = false) {
    const Tile tile = tile_of<16>(p.c, part);
    const int h = part.h;

    const int row = tile.row0 + min(n, tile.rows - 1);
    const int j = divide(row, p.c.div_G), hq = h * p.c.G + row - j * p.c.G;
    const int limit = n < tile.rows ? visible_keys(p.c, tile, j) : 0;
    const int j_last = divide(tile.row0 + tile.rows - 1, p.c.div_G), j_first = divide(tile.row0, p.c.div_G);
    const int limit_max = visible_keys(p.c, tile, j_last);

    Walk<CHOSEN> walk(p, tile, h, j_first, j_last, limit_max, paged_f32_lds + WAVES * stage_bytes(D), tid);
    const int steps = walk.steps();
    const int begin = steps_before(part.from, part.weight, steps), end = steps_before(part.to, part.weight, steps);

    f32m::Rows<D> q, k;
    {
      const float* from = static_cast<const float*>(p.q.data) + (tile.q0 + j) * p.q.token_stride + hq * p.q.head_stride + 4 * g;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) q.v[i] = *reinterpret_cast<const f32x4*>(from + 16 * i);
    }
    const float* const k_pages = static_cast<const float*>(p.k_pages);
    const float* const v_pages = static_cast<const float*>(p.v_pages);
    const char* const stage = paged_f32_lds + wave * stage_bytes(D);
    const Stage keys(stage, lane);
    auto valid_rows = [&](const Granule& at) { return min(max(tile.len - at.pos, 0), GRANULE); };
    auto fetch = [&](const Granule& at) { keys.fill(k_pages + at.row * D, max(valid_rows(at), 1), lane); };

    f32x4 o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const f32m::Exponent prob(p.sm_scale);  // probabilities 2^-8 times: attend_f32.hip
    const float slack = 8.f / prob.up;
    float m = f32m::LOWEST, l = 0.f;

    int it = 2 * begin + wave;
    const int stop = 2 * end;
    Granule at{}, next{};
    if (it < stop) {
      at = walk.locate(it);
      fetch(at);
    }
    for (; it < stop; it += WAVES) {
      const int valid = valid_rows(at);
      const f32m::GlobalBytes vb = f32m::scalar_base(v_pages + at.row * D);
      if (it + WAVES < stop) next = walk.locate(it + WAVES);
      Stage::take(k, stage, lane);
      if (it + WAVES < stop) fetch(next);
      f32x4 v[4][NB / 4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const unsigned off = (max(min(4 * g + r, valid - 1), 0) * D + 4 * n) * 4;
#pragma unroll
        for (int i = 0; i < NB / 4; ++i) v[r][i] = f32m::load16(vb, off + 256 * i);
      }
      f32x4 s = f32m::scores<D>(k, q);
      s *= prob.c;
      const int lim = walk.sees(at, j - j_first) ? limit - at.pos - 4 * g : 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = r < lim ? s[r] : -INFINITY;
      if (valid < GRANULE)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * g + r >= valid)
#pragma unroll
            for (int i = 0; i < NB / 4; ++i) v[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      if (__any(mx > m + slack)) {
        const float m_new = fmaxf(m, f32m::max_groups(mx));
        const float alpha = prob(m, m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] *= alpha;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = prob(s[r], m) * 0x1p-8f;
      l += (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][i / 4][i % 4], s[r], o[i], 0, 0, 0);
      at = next;
    }

    __syncthreads();  // every wavefront has taken its last granule
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
    for (int w = 0; w < WAVES; ++w) l_all += part_l[w][n] * prob(part_m[w][n], m_all);
    const float to_all = prob(m, m_all);
    const float f = !alone ? to_all : l_all > 0.f ? to_all / l_all : l_all;  // nothing seen: zeros; NaN stays
    float* const park = reinterpret_cast<float*>(paged_f32_lds);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NB / 4; ++i) {  // lane (n, g) holds columns 64 i + 16 g + 4 r + (0..3) of query n
        const f32x4 x = {o[4 * i][r], o[4 * i + 1][r], o[4 * i + 2][r], o[4 * i + 3][r]};
        *reinterpret_cast<f32x4*>(park + (wave * 16 + n) * PITCH + 64 * i + 16 * g + 4 * r) = x * f;
      }
    if (wave == 0 && g == 0 && n < tile.rows) {
      const long long out_row = static_cast<long long>(tile.q0 + j) * p.c.Hq + hq;
      if (!alone) {
        float* to = p.parts.ml + (part_base + n) * 2;
        to[0] = m_all;
        to[1] = l_all;
      } else if (p.lse) {
        p.lse[out_row] = natural_lse_f32(m_all, l_all, prob);
      }
    }
    __syncthreads();
    for (int e = tid; e < tile.rows * (D / 4); e += 64 * WAVES) {
      const int r = e / (D / 4), col = e % (D / 4) * 4;
      f32x4 x = *reinterpret_cast<const f32x4*>(park + r * PITCH + col);
#pragma unroll
      for (int w = 1; w < WAVES; ++w) x += *reinterpret_cast<const f32x4*>(park + (w * 16 + r) * PITCH + col);
      const int jr = divide(tile.row0 + r, p.c.div_G), hr = h * p.c.G + tile.row0 + r - jr * p.c.G;
      float* to = alone ? static_cast<float*>(const_cast<void*>(p.out.data)) + (tile.q0 + jr) * p.out.token_stride +
                              hr * p.out.head_stride + col
                        : p.parts.o + (part_base + r) * D + col;
      *reinterpret_cast<f32x4*>(to) = x;
      if (x[0] != x[0] || x[1] != x[1] || x[2] != x[2] || x[3] != x[3]) atomicOr(&nan_rows, 1u << r);
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
      for (int i = 0; i < WAVES; ++i) l_row += part_l[i][r] * prob(part_m[i][r], m_row);
      const float norm = !alone ? 1.f : l_row > 0.f ? 1.f / l_row : l_row;
      float* const to = !alone ? z.parts.o + (part_base + r) * D
                               : static_cast<float*>(const_cast<void*>(z.out.data)) + (tile.q0 + jr) * z.out.token_stride + hr * z.out.head_stride;
      redo_row<float, NATIVE, D, CHOSEN>(
          z, tile.q0 + jr, hr, visible_keys(z.c, tile, jr), tile.len, 2 * begin, 2 * end, false,
          [&](int gr) {
            const Granule x = walk.locate(gr);
            return RedoGranule{x.row, x.pos, walk.sees(x, jr - j_first)};
          },
          [&](float score) { return prob(score * prob.c, m_row) * 0x1p-8f; },
          [&](int col) { return to[col]; }, [&](int col, float x, float) { to[col] = x * norm; });
    }
    if (CHOSEN) __syncthreads();  // the walk's tables are free as well
  }
}

template <int D, bool CHOSEN>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  const size_t lds = WAVES * stage_bytes(D) + (CHOSEN ? walk_lds_bytes(p) : 0);
  static std::atomic<unsigned long long> allowed{0};
  if (lds > 64 * 1024)
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(&paged_attend_f32_kernel<D, CHOSEN>), WALK_LDS, allowed)) return e;
  hipLaunchKernelGGL((paged_attend_f32_kernel<D, CHOSEN>), dim3(p.parts.grid), dim3(64 * WAVES), lds, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attend_f32(const PagedAttendParams& p, int d, hipStream_t stream) {
  if (p.selected) return d == 128 ? launch<128, true>(p, stream) : launch<64, true>(p, stream);
  return d == 128 ? launch<128, false>(p, stream) : launch<64, false>(p, stream);
}

}  // namespace heatkv
