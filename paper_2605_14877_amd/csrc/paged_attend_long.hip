// Attention of new tokens over the paged cache, bf16, for requests with many query rows (chunks of prompts, whole scales):
// the tile loop of attend.hip over keys that lie on pages.
//
// Workgroup = 4 wavefronts x 32 query rows (row = token x query of the kv head's group), two workgroups per compute unit.
// The request's keys are walked in tiles of 64, four granules of 16 rows, each with an address of its own; tile format,
// copies and operand layouts are those of tile_lds.h.  Rows behind the request's end arrive as zeros (range-checked
// copies), keys that a row does not see get a score of -inf in the tiles where that can be.
// 8-bit cache rows come through registers, converted on the way into the stage.
//
// Bound: the matrix pipe, and the vector work of the softmax next to it.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "paged.h"
#include "paged_schedule.h"
#include "paged_walk.h"
#include "tile_lds.h"

namespace heatkv {

namespace {

using namespace paged;

constexpr int BM = 128, BN = tile::ROWS;  // query rows of a workgroup, keys of a tile
extern __shared__ __attribute__((aligned(1024))) char paged_long_lds[];

__device__ __forceinline__ uint4 codes_to_chunk(unsigned lo, unsigned hi) {  // 8 E4M3 codes as bf16 (exact)
  union {
    bf16x2 h[4];
    uint4 u;
  } o;
  o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(lo), 1.0f, false);
  o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(lo), 1.0f, true);
  o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(hi), 1.0f, false);
  o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(hi), 1.0f, true);
  return o.u;
}

template <int D, bool FP8>
__global__ __launch_bounds__(256, 2) void paged_attend_long_kernel(AttendParams p) {
  constexpr int RB = 2 * D, TILE_BYTES = BN * RB, SRC = FP8 ? D : RB;
  constexpr int NK = D / 16, NV = D / 32;
  constexpr int CPT = TILE_BYTES / 4096;            // copies of a tile per wavefront (bf16 rows)
  constexpr int CPL = BN * D / 16 / 256;            // 16-byte loads of a tile per lane (8-bit rows)
  char(*const lds)[2][TILE_BYTES] = reinterpret_cast<char(*)[2][TILE_BYTES]>(paged_long_lds);  // [stage][K, V]

  __shared__ Scratch scratch;

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = blockIdx.x;
  Place place = find_place<BM, BN>(p, w, scratch);
  write_border(p, place, w);
  Part part;
  while (next_part<BM, BN>(p, place, part)) {
  const Tile tl = tile_of<BM>(p.c, part);
  const int h = part.h;
  const int j_last = divide(tl.row0 + tl.rows - 1, p.c.div_G);
  const int steps = (visible_keys(p.c, tl, j_last) + BN - 1) / BN;
  const int begin = steps_before(part.from, part.weight, steps), end = steps_before(part.to, part.weight, steps);
  const bool alone = part.from == 0 && part.to == part.weight;

  // Rows of this wavefront; one without rows still copies its share of the tiles.
  const int w_row = wave * 32;
  const bool active = w_row < tl.rows;
  const int row = tl.row0 + min(w_row + n, tl.rows - 1);
  const int j = divide(row, p.c.div_G), hq = h * p.c.G + row - j * p.c.G;
  const bool real = w_row + n < tl.rows;
  const int limit = real ? visible_keys(p.c, tl, j) : 0;
  const int limit_min = w_row + 32 <= tl.rows ? visible_keys(p.c, tl, divide(tl.row0 + w_row, p.c.div_G)) : 0;
  const int limit_max = active ? visible_keys(p.c, tl, divide(tl.row0 + min(w_row + 31, tl.rows - 1), p.c.div_G)) : 0;

  bf16x8 qreg[NK];
  {
    const bf16_t* from = static_cast<const bf16_t*>(p.q.data) + (tl.q0 + j) * p.q.token_stride + hq * p.q.head_stride + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) qreg[ks] = *reinterpret_cast<const bf16x8*>(from + 16 * ks);
  }

  const long long table = static_cast<long long>(tl.b) * p.c.max_pages;
  const char* const k_pages = static_cast<const char*>(p.k_pages);
  const char* const v_pages = static_cast<const char*>(p.v_pages);
  // Byte offset of the cache row at position x (a multiple of 16 below the request's end).
  auto row_at = [&](int x) {
    return (page_row(p.c, uniform_load(p.c.table, table + (x >> p.c.page_log2)), h) + (x & ((1 << p.c.page_log2) - 1))) * SRC;
  };

  const int ld_off_k = tile::loader_off_k<RB>(wave, lane), ld_off_v = tile::loader_off_v<RB>(wave, lane);
  const unsigned lds_base = static_cast<unsigned>(reinterpret_cast<unsigned long long>(
      (__attribute__((address_space(3))) char*)(paged_long_lds)));
  const unsigned lds_wave = __builtin_amdgcn_readfirstlane(lds_base + wave * 1024);
  // bf16 rows: this wavefront's copies of tile `it` into a stage.  Copy i covers rows (64 / CPT) i + (16 / CPT) wave of the
  // tile and on, all of one granule.
  auto copy_tile = [&](int it, auto buf_tag) {
    constexpr int buf = decltype(buf_tag)::value;
    constexpr int PER = 64 / CPT;  // rows between copies of a wavefront
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int ahead = PER == 32 ? 16 * (wave >> 1) : 0;  // rows of the lane offset that belong to the granule's place
      const int x = it * BN + PER * i + ahead;
      const int left = tl.len - x;
      const long long at = (left > 0 ? row_at(x) : 0) - ahead * RB;
      const int rows = left > 0 ? left + ahead : 0;
      tile::copy_1k_checked(lds_wave, buf * (2 * TILE_BYTES) + 4096 * i, ld_off_k, tile::tile_descriptor<RB>(k_pages + at, rows), 0);
      tile::copy_1k_checked(lds_wave, buf * (2 * TILE_BYTES) + TILE_BYTES + 4096 * i, ld_off_v,
                            tile::tile_descriptor<RB>(v_pages + at, rows), 0);
    }
  };
  // 8-bit rows: load i of a lane is 16 codes of one row.
  constexpr int LPR = D / 16;  // lanes per row
  uint4 raw_k[CPL], raw_v[CPL];
  auto load_codes = [&](int it) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int r = (tid + 256 * i) / LPR;
      const int gr = __builtin_amdgcn_readfirstlane(r / 16);  // a wavefront's 64 / LPR rows are in one granule
      const int x = it * BN + 16 * gr;
      raw_k[i] = raw_v[i] = make_uint4(0, 0, 0, 0);
      if (x < tl.len) {
        const long long at = row_at(x) + (r % 16) * SRC + (tid % LPR) * 16;
        if (x + r % 16 < tl.len) {
          raw_k[i] = ldg16(k_pages + at);
          raw_v[i] = ldg16(v_pages + at);
        }
      }
    }
  };
  auto store_codes = [&](int buf) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int r = (tid + 256 * i) / LPR, chunk = 2 * (tid % LPR);
      const int sk = tile::swizzle_k<RB>(r & 15), sv = tile::swizzle_v<RB>(r & 15);
      char* kt = lds[buf][0] + r * RB;
      char* vt = lds[buf][1] + r * RB;
      *reinterpret_cast<uint4*>(kt + ((chunk ^ sk) << 4)) = codes_to_chunk(raw_k[i].x, raw_k[i].y);
      *reinterpret_cast<uint4*>(kt + (((chunk + 1) ^ sk) << 4)) = codes_to_chunk(raw_k[i].z, raw_k[i].w);
      *reinterpret_cast<uint4*>(vt + ((chunk ^ sv) << 4)) = codes_to_chunk(raw_v[i].x, raw_v[i].y);
      *reinterpret_cast<uint4*>(vt + (((chunk + 1) ^ sv) << 4)) = codes_to_chunk(raw_v[i].z, raw_v[i].w);
    }
  };
  int k_off[NK], v_off[NV];
  tile::reader_off_k<RB>(lane, k_off);
  tile::reader_off_v<RB>(lane, v_off);

  f32x16 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  const float c = p.sm_scale * kLog2e;
  float m = lowest_reference(c), l = 0.f;
  constexpr float kSlack = 8.f;  // attend.hip
  const float slack = kSlack / c;

  auto math = [&](int it, auto buf_tag) {
    constexpr int buf = decltype(buf_tag)::value;
    const char* kt = lds[buf][0];
    const char* vt = lds[buf][1];
    f32x16 s[2];
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[cb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int cb = 0; cb < 2; ++cb) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(kt + cb * 32 * RB + k_off[ks]);
        s[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[ks], s[cb], 0, 0, 0);
      }
    if (it * BN + BN > limit_min) tile::mask_rows(limit - it * BN, hl, s);
    float mx = s[0][0];
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[cb][r]);
    mx = max_halves(mx);
    if (__any(mx > m + slack)) {
      const float m_new = fmaxf(m, mx);
      const float alpha = fast_exp2((m - m_new) * c);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
    }
    const float mc = m * c;
#pragma unroll
    for (int chunk = 0; chunk < 4; ++chunk) {
      union VOperand {
        struct {
          s16x4 lo, hi;
        } s;
        bf16x8 v;
      } va[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const char* base = vt + 16 * chunk * RB + v_off[i];
        va[i].s.lo = lds_read_tr16(reinterpret_cast<const bf16_t*>(base));
        va[i].s.hi = lds_read_tr16(reinterpret_cast<const bf16_t*>(base + 8 * RB));
      }
      bf16x8 pb;  // rounded for the product; the row sum takes them as they are (its logarithm is an output, in fp32)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = fast_exp2(fmaf(s[chunk >> 1][8 * (chunk & 1) + i], c, -mc));
        l += e;
        pb[i] = static_cast<bf16_t>(e);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[i].v, pb, o[i], 0, 0, 0);
    }
  };

  // Stage b holds tile begin + 2 x + b.  One barrier a tile: the copies of tile `it` have landed for all, and the stage
  // that the next copies go to has been read by all.
  auto step = [&](int it, auto buf_tag) {
    constexpr int buf = decltype(buf_tag)::value;
    wait_vmcnt<0>();
    __syncthreads();
    const bool more = it + 1 < end;
    if (more) {
      if constexpr (FP8)
        load_codes(it + 1);
      else
        copy_tile(it + 1, std::integral_constant<int, 1 - buf>{});
    }
    if (active && it * BN < limit_max) math(it, buf_tag);
    if constexpr (FP8)
      if (more) store_codes(1 - buf);
  };
  if (begin < end) {
    if constexpr (FP8) {
      load_codes(begin);
      store_codes(0);
    } else {
      copy_tile(begin, std::integral_constant<int, 0>{});
    }
  }
  int it = begin;
  for (; it + 1 < end; it += 2) {
    step(it, std::integral_constant<int, 0>{});
    step(it + 1, std::integral_constant<int, 1>{});
  }
  if (it < end) step(it, std::integral_constant<int, 0>{});

  // Lane (n, hl) holds columns 32 i + 8 (r / 4) + 4 hl + r % 4 of query n.
  l = sum_halves(l);
  if (real) {
  const long long out_row = static_cast<long long>(tl.q0 + j) * p.c.Hq + hq;
  const long long part_row = part_rows<BM>(w, part.from == 0) + w_row + n;
  if (hl == 0) {
    if (!alone) {
      p.part_ml[part_row * 2] = m;
      p.part_ml[part_row * 2 + 1] = l;
    } else if (p.lse) {
      p.lse[out_row] = natural_lse(m, l, p.sm_scale);
    }
  }
  if (!alone) {
    float* to = p.part_o + part_row * D + 4 * hl;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4*>(to + 32 * i + 8 * r) = f32x4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
  } else {
    const float f = l > 0.f ? 1.f / l : l;  // nothing seen: zeros; NaN stays
    bf16_t* to = static_cast<bf16_t*>(const_cast<void*>(p.out.data)) + (tl.q0 + j) * p.out.token_stride +
                 hq * p.out.head_stride + 4 * hl;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        bf16x4 y;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = static_cast<bf16_t>(o[i][4 * r + k] * f);
        *reinterpret_cast<bf16x4*>(to + 32 * i + 8 * r) = y;
      }
  }
  }
  __syncthreads();  // the stages are free for the next segment
  }
}

template <int D, bool FP8>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((paged_attend_long_kernel<D, FP8>), dim3(p.grid), dim3(256), 4 * BN * 2 * D, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attend_long(const PagedAttendParams& p, int d, bool fp8, hipStream_t stream) {
  if (d == 128) return fp8 ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
  return fp8 ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
}

}  // namespace heatkv
