// Attention of new tokens over the paged cache, bf16, for requests with many query rows (chunks of prompts, whole scales):
// the tile loop of attend.hip over keys that lie on pages.
//
// The grid has the workgroups of the 16-row kernel as well (place_of_few()).
//
// Workgroup = 4 wavefronts x 32 query rows (row = token x query of the kv head's group), two workgroups per compute unit (4-bit rows at
// d = 64: three).
// The request's keys are walked in tiles of 64, four granules of 16 rows, each with an address of its own; tile format,
// copies and operand layouts are those of tile_lds.h.  Rows behind the request's end arrive as zeros (range-checked
// copies), keys that a row does not see get a score of -inf in the tiles where that can be.
// 8-bit and 4-bit cache rows come through registers, converted on the way into the stage.
// Chosen pages: the walk is over the union of the pages that the workgroup's tokens have chosen (up to 128 of them, neighbours in
// the request, which choose alike), with a word of 32 tokens for each wavefront and page.
//
// Bound: the matrix pipe, and the vector work of the softmax next to it.  2 x 2048 new tokens over 4096 keys before them, 32 heads over 8,
// d = 128: 344 GFLOP in 335 us, 1.0 PFLOP/s (385 us where the clock falls under the load of many in a row); 8-bit rows 3 % more, for their
// way through registers, 4-bit rows no more.  Whole scales of 8 requests, 16 heads, d = 64, 11520 tile steps: 46 us, no pipe full (4-bit
// rows: vector work 21 %, matrix pipe 18 %, waiting 37 %, for issue 30 %), 368 tiles cut for 768 places.  Chosen pages, 1024 tokens, 32 of
// 272 pages each, 127 in the union of 32 tokens: 96 us, as much as the union's products (57 GFLOP) at 0.6 PFLOP/s.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.h"
#include "paged.h"
#include "paged_attend_few.h"
#include "paged_redo.h"
#include "paged_rules.h"
#include "paged_schedule.h"
#include "paged_walk.h"
#include "tile_lds.h"

namespace heatkv {

namespace {

using namespace paged;

constexpr int BM = 128, BN = tile::ROWS;  // query rows of a workgroup, keys of a tile
extern __shared__ __attribute__((aligned(1024))) char paged_long_lds[];

// Where the four granules of a tile lie, in granules of the cache (there are less than 2^31, check_shape()).
struct TileRows {
  int granule[4];
  int pos[4];  // chosen pages: position of the first key
};

// The union of a tile's chosen pages, in LDS behind the stages: `count`, a bit for each page of the request, how many there are
// in the words before, and for each page of the union where it lies (granule of the cache), its first position / page size, and
// who has chosen it.
struct Union {
  int* count;
  unsigned* bits;
  int *before, *granule, *page;
  unsigned* who;  // [pages][4]: bit i = token i of the wavefront's tokens
  __device__ __forceinline__ Union(char* lds, int max_pages, int capacity) {
    const int words = (max_pages + 31) / 32;
    count = reinterpret_cast<int*>(lds);
    bits = reinterpret_cast<unsigned*>(lds + 16);
    before = reinterpret_cast<int*>(bits + words);
    granule = before + words;
    page = granule + capacity;
    who = reinterpret_cast<unsigned*>(page + capacity);
  }
};

__device__ __forceinline__ const __attribute__((address_space(3))) char* lds_pointer(int at) {
  return (const __attribute__((address_space(3))) char*)static_cast<size_t>(static_cast<unsigned>(at));
}

__device__ __forceinline__ int pick(int which, int one, int other) {
  int x;
  asm("s_cmp_lg_u32 %1, 0\n\ts_cselect_b32 %0, %2, %3" : "=s"(x) : "s"(which), "s"(one), "s"(other) : "scc");
  return x;
}

// Codes of a lane's load of a 4-bit row, and their scale byte.
struct Nibbles {
  uint4 w;
  unsigned char scale;
};

struct Shared {
  Scratch scratch;
  Part piece;
};
constexpr size_t kUnionAt = (sizeof(Shared) + 15) / 16 * 16;  // behind the stages

// Fills the union, by all lanes; returns its size.  Entries of a token lie H * top apart.
__device__ __forceinline__ int build_union(const AttendParams& a, const Tile& t, int h, int j_first, int j_last, int seen_last,
                                           const Union& u, int capacity) {
  const Cache& c = a.c;
  const int tid = threadIdx.x, words = (c.max_pages + 31) / 32, per_log2 = c.page_log2 - 4;
  for (int i = tid; i < words; i += 256) u.bits[i] = 0;
  for (int i = tid; i < 4 * capacity; i += 256) u.who[i] = 0;
  __syncthreads();
  const int seen = (seen_last + (1 << c.page_log2) - 1) >> c.page_log2, entries = (j_last - j_first + 1) * a.top;
  auto entry = [&](int i, int& token) {
    token = i / a.top;
    const int x = a.selected[((static_cast<long long>(t.q0) + j_first + token) * c.H + h) * a.top + i - token * a.top];
    return x < seen ? x : -1;
  };
  for (int i = tid; i < entries; i += 256) {
    int token;
    const int x = entry(i, token);
    if (x >= 0) atomicOr(&u.bits[x >> 5], 1u << (x & 31));
  }
  __syncthreads();
  if (tid < 64) {
    const int total = scan_bits(u.bits, u.before, words, tid);
    if (tid == 0) *u.count = total;
  }
  __syncthreads();
  for (int i = tid; i < entries; i += 256) {
    int token;
    const int x = entry(i, token);
    if (x < 0) continue;
    const int at = u.before[x >> 5] + __popc(u.bits[x >> 5] & ((1u << (x & 31)) - 1));
    const unsigned e = min(static_cast<unsigned>(c.table[static_cast<long long>(t.b) * c.max_pages + x]),
                           static_cast<unsigned>(c.num_pages - 1));
    u.page[at] = x;
    u.granule[at] = (static_cast<int>(e) * c.H + h) << per_log2;
    // the wavefronts that have rows of the token: one, or two where the group does not divide 32
    const int row = (j_first + token) * c.G - t.row0, first = max(row, 0) / 32, last = min(row + c.G - 1, BM - 1) / 32;
    for (int w = first; w <= last; ++w)
      atomicOr(&u.who[4 * at + w], 1u << (j_first + token - divide(t.row0 + 32 * w, c.div_G)));
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*u.count);
}

// 4-bit rows at d = 64 take 176 registers by themselves; held to 168, three workgroups share a compute unit instead of two: whole scales of 8
// requests 59 us instead of 68, 3000 new tokens over 4096 keys 178 instead of 206, 16 x 300 228 instead of 252; where two to a unit come
// out even, 230 instead of 222 (2 x 2048); all with the 16-row kernel in a launch of its own.
// few: the 16-row kernel's launch (paged_attend_few.h), whose workgroups are the grid's from few_at on, 0 or behind this kernel's own, or
// none.  As a launch of its own it took 4 to 8 us where it had next to nothing to do, and what it did have did not run beside this.
template <int D, Format F, bool CHOSEN>
__global__ __launch_bounds__(256, D == 64 && F == E2M1 ? 3 : 2) void paged_attend_long_kernel(AttendParams p, AttendParams few, int few_at) {
  int w = blockIdx.x;
  if (static_cast<unsigned>(w - few_at) < static_cast<unsigned>(few.parts.grid)) {
    constexpr int STAGES = FEW_WAVES * stage_bytes(D);
    return attend_few<D, F, CHOSEN, 1>(few, w - few_at, *reinterpret_cast<FewShared*>(paged_long_lds + STAGES), paged_long_lds,
                                       paged_long_lds + STAGES + FEW_SHARED);
  }
  if (few_at == 0) w -= few.parts.grid;
  constexpr bool CODES = F == E4M3, FP4 = F == E2M1;
  constexpr int RB = 2 * D, TILE_BYTES = BN * RB, SRC = row_bytes<bf16_t, F>(D);
  constexpr int NK = D / 16, NV = D / 32;
  constexpr int CPT = TILE_BYTES / 4096;            // copies of a tile per wavefront (bf16 rows)
  constexpr int CPL = BN * D / 16 / 256;            // 16-byte loads of a tile per lane (8-bit rows)
  char(*const lds)[2][TILE_BYTES] = reinterpret_cast<char(*)[2][TILE_BYTES]>(paged_long_lds);  // [stage][K, V]
  // Behind the stages, which then begin at LDS address 0: all of their offsets fit into the read instructions.
  Shared& shared = *reinterpret_cast<Shared*>(paged_long_lds + 4 * TILE_BYTES);

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned lds_base = static_cast<unsigned>(reinterpret_cast<unsigned long long>(
      (__attribute__((address_space(3))) char*)(paged_long_lds)));
  const unsigned lds_wave = __builtin_amdgcn_readfirstlane(lds_base + wave * 1024);
  const int ld_off_k = tile::loader_off_k<RB>(wave, lane), ld_off_v = tile::loader_off_v<RB>(wave, lane);
  // Reader offsets as LDS addresses: stage, tile and row of a read are then constants of the instruction.
  int k_off[NK], v_off[NV];
  tile::reader_off_k<RB>(lane, k_off);
  tile::reader_off_v<RB>(lane, v_off);
#pragma unroll
  for (int i = 0; i < NK; ++i) k_off[i] += lds_base;
#pragma unroll
  for (int i = 0; i < NV; ++i) v_off[i] += lds_base;
  const char* const k_pages = static_cast<const char*>(p.k_pages);
  const char* const v_pages = static_cast<const char*>(p.v_pages);
  const float c = p.sm_scale * kLog2e;
  constexpr float kSlack = 8.f;  // the reference is raised by more than this only: attend.hip
  const float slack = kSlack / c;

  // The piece at hand stays in LDS, and arguments are read where they are used: the tile loop has no registers to keep them in.
  {
    Part part;
    if (!only_piece<BM, BN>(p, w, shared.scratch, part)) return;
    if (tid == 0) shared.piece = part;
    __syncthreads();
  }
  const AttendParams& a = arguments();
  const Part part{__builtin_amdgcn_readfirstlane(shared.piece.b), __builtin_amdgcn_readfirstlane(shared.piece.h),
                  __builtin_amdgcn_readfirstlane(shared.piece.t), uniform(shared.piece.from), uniform(shared.piece.to),
                  uniform(shared.piece.weight)};
  const Tile tl = tile_of<BM>(a.c, part);
  const int h = part.h;
  const int j_first = divide(tl.row0, a.c.div_G), j_last = divide(tl.row0 + tl.rows - 1, a.c.div_G);
  const int seen_last = visible_keys(a.c, tl, j_last);
  const int capacity = CHOSEN ? many_capacity(a.c, a.top) : 0;
  const Union chosen(paged_long_lds + 4 * TILE_BYTES + kUnionAt, a.c.max_pages, capacity);
  int steps = (seen_last + BN - 1) / BN, n_pages = 0;
  if constexpr (CHOSEN) {
    n_pages = build_union(a, tl, h, j_first, j_last, seen_last, chosen, capacity);
    steps = ((n_pages << (a.c.page_log2 - 4)) + 3) / 4;
  }
  const int begin = steps_before(part.from, part.weight, steps), end = steps_before(part.to, part.weight, steps);

  // Rows of this wavefront; one without rows still copies its share of the tiles.
  const int w_row = wave * 32;
  const bool active = w_row < tl.rows;
  const int limit_min = w_row + 32 <= tl.rows ? visible_keys(a.c, tl, divide(tl.row0 + w_row, a.c.div_G)) : 0;
  const int limit_max = active ? visible_keys(a.c, tl, divide(tl.row0 + min(w_row + 31, tl.rows - 1), a.c.div_G)) : 0;
  // Tiles that this wavefront has to do with.
  const int my_end = CHOSEN ? (active ? end : begin) : min(end, (limit_max + BN - 1) / BN);
  [[maybe_unused]] const int w_first = divide(tl.row0 + w_row, a.c.div_G);  // the wavefront's token 0
  struct Row {
    int j, hq;  // token of the request, query head
    bool real;
  };
  auto row_of = [&](const AttendParams& a) {
    const int row = tl.row0 + min(w_row + n, tl.rows - 1), j = divide(row, a.c.div_G);
    return Row{j, h * a.c.G + row - j * a.c.G, w_row + n < tl.rows};
  };
  const Row my = row_of(a);
  [[maybe_unused]] const int token = my.j - w_first;
  const int limit = my.real ? visible_keys(a.c, tl, my.j) : 0;
  // Table row of the request; page size in granules.
  const int* const table = a.c.table + static_cast<long long>(tl.b) * a.c.max_pages;
  const int per_log2 = a.c.page_log2 - 4, heads = a.c.H, last_page = a.c.num_pages - 1;
  struct Place {
    int granule, pos;
  };
  auto locate_granule = [&](int g) {  // of the walk
    if constexpr (CHOSEN) {
      const int u = min(g >> per_log2, n_pages - 1), off = g & ((1 << per_log2) - 1);
      return Place{__builtin_amdgcn_readfirstlane(chosen.granule[u]) + off,
                   (g >> per_log2) < n_pages ? ((__builtin_amdgcn_readfirstlane(chosen.page[u]) << per_log2) + off) * 16 : 1 << 30};
    }
    const int x = min(g, max(tl.len - 1, 0) >> 4);  // granule of the request
    const unsigned e = min(static_cast<unsigned>(uniform_load(table, x >> per_log2)), static_cast<unsigned>(last_page));
    return Place{((static_cast<int>(e) * heads + h) << per_log2) + (x & ((1 << per_log2) - 1)), 16 * g};
  };
  auto locate = [&](int it) {
    TileRows r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Place x = locate_granule(4 * it + i);
      r.granule[i] = x.granule;
      r.pos[i] = x.pos;
    }
    return r;
  };

  bf16x8 qreg[NK];
  {
    const bf16_t* from = static_cast<const bf16_t*>(a.q.data) + (tl.q0 + my.j) * a.q.token_stride + my.hq * a.q.head_stride + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) qreg[ks] = *reinterpret_cast<const bf16x8*>(from + 16 * ks);
  }

  // A tile behind the part's end has no rows: its copies touch no memory.
  const int stop = CHOSEN ? tl.len : min(tl.len, end * BN);
  // bf16 rows: copy i of this wavefront of a K or V tile covers rows (64 / CPT) i + (16 / CPT) wave and on, all of one
  // granule; rows behind the request's end arrive as zeros (a probability of 0 does not remove an infinity).
  auto source = [&](const char* pages, const TileRows& at, int it, int i) {
    constexpr int PER = 64 / CPT;                        // rows between copies of a wavefront
    const int ahead = PER == 16 ? 0 : 16 * (wave >> 1);  // rows of the lane offset that belong to the granule's place
    const int gr = PER == 16 ? i : 2 * i;                // granule of the lane offset's row 0, but for `ahead`
    const int left = CHOSEN ? (it < end ? stop + ahead - (PER == 16 ? at.pos[gr] : wave >> 1 ? at.pos[gr + 1] : at.pos[gr]) : 0)
                            : stop - it * BN - PER * i;  // valid rows from those of the lane offset's row 0 on
    const int from = PER == 16 ? at.granule[i] : wave >> 1 ? at.granule[2 * i + 1] : at.granule[2 * i];
    return tile::tile_descriptor<RB>(pages + (static_cast<long long>(from) * 16 - ahead) * RB, left > ahead ? left : 0);
  };
  auto copy_k = [&](const TileRows& at, int it, auto buf_tag, int i) {
    tile::copy_1k_checked(lds_wave, decltype(buf_tag)::value * (2 * TILE_BYTES) + 4096 * i, ld_off_k, source(k_pages, at, it, i), 0);
  };
  auto copy_v = [&](const TileRows& at, int it, auto buf_tag, int i) {
    tile::copy_1k_checked(lds_wave, decltype(buf_tag)::value * (2 * TILE_BYTES) + TILE_BYTES + 4096 * i, ld_off_v,
                          source(v_pages, at, it, i), 0);
  };
  // 8-bit rows: load i of a lane is 16 codes of one row, converted on the way into the stage.
  constexpr int LPR = D / 16;  // lanes per row
  // Row and place within a granule, the same for all of a lane's loads.  As an address for each load they went to scratch, and their reload
  // waited for the load before it: 2 x 2048 tokens over 4096 keys 377 us instead of 354, 3000 tokens 347 instead of 299.
  const int code_row = tid / LPR & 15, code_at = code_row * SRC + tid % LPR * 16;
  auto load_codes = [&](const char* pages, const TileRows& at, int it, int i) {
    const int r = (tid + 256 * i) / LPR;  // a wavefront's 64 / LPR rows are of one granule
    // By arithmetic on all four places: a choice of one in memory would keep them there.
    auto mine = [&](const int (&x)[4]) {
      const int x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
      if constexpr (D == 64) return pick(wave >> 1, pick(wave & 1, x3, x2), pick(wave & 1, x1, x0));
      return i ? pick(wave >> 1, x3, x2) : pick(wave >> 1, x1, x0);
    };
    [[maybe_unused]] const int here = mine(at.pos);  // for any `it`: no branch around it within the step
    const int from = mine(at.granule);
    const int pos = !CHOSEN ? it * BN + (r & ~15) : it >= end ? 1 << 30 : here;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (pos + code_row < stop) raw = ldg16(pages + static_cast<long long>(from) * (16 * SRC) + code_at);
    return raw;
  };
  auto store_codes = [&](char* stage, const uint4& raw, int i, auto is_v) {
    const int r = (tid + 256 * i) / LPR, chunk = 2 * (tid % LPR);
    const int swz = decltype(is_v)::value ? tile::swizzle_v<RB>(r & 15) : tile::swizzle_k<RB>(r & 15);
    *reinterpret_cast<bf16x8*>(stage + r * RB + ((chunk ^ swz) << 4)) = codes_to_bf16(raw.x, raw.y);
    *reinterpret_cast<bf16x8*>(stage + r * RB + (((chunk + 1) ^ swz) << 4)) = codes_to_bf16(raw.z, raw.w);
  };
  // 4-bit rows: a wavefront has one granule of the tile, a lane D / 4 codes of one row and their scale byte.
  auto locate_own = [&](int it) { return locate_granule(4 * it + wave); };
  auto load_nibbles = [&](const char* pages, const Place& at) {
    const char* const first = pages + static_cast<long long>(at.granule) * (16 * SRC);
    Nibbles raw{make_uint4(0, 0, 0, 0), static_cast<unsigned char>(first[8 * D + lane * D / 128])};
    if constexpr (D == 128) {
      raw.w = ldg16(first + lane * 16);
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(first + lane * 8);
      raw.w.x = w.x;
      raw.w.y = w.y;
    }
    return raw;
  };
  // K: rows that no row of queries sees may be anything, their scores are replaced.  V: rows behind the request's end have to be zeros.
  auto load_v_nibbles = [&](const Place& at, int it) {
    const int left = stop - (it >= end ? 1 << 30 : at.pos);
    Nibbles raw{make_uint4(0, 0, 0, 0), 127};
    if (left >= 16) {
      raw = load_nibbles(v_pages, at);
    } else if (lane / 4 < left) {
      raw = load_nibbles(v_pages, at);
    }
    return raw;
  };
  // Chunk i of a lane's D / 32: 8 columns.  The swizzle of V leaves the chunks of a lane side by side, that of K does not.
  const int nibble_row = 16 * wave + lane / 4, nibble_chunk = D / 32 * (lane % 4);
  const int k_to = nibble_row * RB + ((nibble_chunk ^ tile::swizzle_k<RB>(nibble_row & 15)) << 4);
  const int v_to = nibble_row * RB + ((nibble_chunk ^ tile::swizzle_v<RB>(nibble_row & 15)) << 4);
  auto store_nibbles = [&](char* stage, const Nibbles& raw, int i, auto is_v) {
    const unsigned w = i == 0 ? raw.w.x : i == 1 ? raw.w.y : i == 2 ? raw.w.z : raw.w.w;
    const int to = decltype(is_v)::value ? v_to + 16 * i : k_to ^ 16 * i;
    *reinterpret_cast<bf16x8*>(stage + to) = nibbles_to_bf16(w, scale_of(raw.scale));
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;

  f32x16 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  float m = lowest_reference(c), l = 0.f;

  union VOperand {
    struct {
      s16x4 lo, hi;
    } s;
    bf16x8 v;
  };
  // Operands out of a stage: K rows 32 cb + n, step ks; V columns 32 i + .., keys 16 chunk + ..
  auto read_k = [&](auto buf_tag, int ks, int cb) {
    return *(const __attribute__((address_space(3))) bf16x8*)(lds_pointer(k_off[ks]) +
                                                              (decltype(buf_tag)::value * (2 * TILE_BYTES) + cb * 32 * RB));
  };
  auto read_v = [&](auto buf_tag, int chunk, int i) {
    const auto* at = lds_pointer(v_off[i]) + (decltype(buf_tag)::value * (2 * TILE_BYTES) + TILE_BYTES + 16 * chunk * RB);
    VOperand x;
    x.s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)at);
    x.s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at + 8 * RB));
    return x.v;
  };
  // S^T = K Q^T of the 64 keys of a K tile.
  auto scores = [&](f32x16 (&s)[2], auto buf_tag) {
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[cb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int cb = 0; cb < 2; ++cb)
        s[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(buf_tag, ks, cb), qreg[ks], s[cb], 0, 0, 0);
  };
  auto lane_max = [&](const f32x16 (&s)[2]) {
    float mx = s[0][0];
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[cb][r]);
    return mx;
  };
  auto raise = [&](float mx) {
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
  };
  // Masks what a row of tile `it` does not see; whether there may be such.
  auto mask = [&](int it, f32x16 (&s)[2]) {
    if constexpr (CHOSEN) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // s[i / 2][8 (i % 2) + r] is key 8 (r / 4) + 4 hl + r % 4 of granule i
        const int g = 4 * it + i, u = min(g >> per_log2, n_pages - 1), off = g & ((1 << per_log2) - 1);
        const int pos = ((chosen.page[u] << per_log2) + off) * 16;
        const bool sees = (g >> per_log2) < n_pages && (chosen.who[4 * u + wave] >> token & 1);
        int lim = (sees ? limit - pos : 0) - 4 * hl;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int at = 8 * (i & 1) + r;
          s[i >> 1][at] = 8 * (r >> 2) + (r & 3) < lim ? s[i >> 1][at] : -INFINITY;
        }
      }
      return true;
    }
    if (it * BN + BN <= limit_min) return false;
    tile::mask_rows(limit - it * BN, hl, s);
    return true;
  };
  // Masks tile `it`, of whose scores `mx` is the lane's maximum; the maximum of those that are seen.  Chosen pages: where
  // the tile lies in one page and ends before the last key of all rows, a row sees all of it or nothing.  `open` is whether
  // it does, and takes the scores' place: behind a closed one the probabilities are 2^(s c - inf) = 0, or NaN where s is not
  // finite; the row is then done anew (paged_redo.h).
  auto seen_max = [&](int it, f32x16 (&s)[2], float mx, bool& open) {
    if constexpr (CHOSEN) {
      if (per_log2 >= 2) {
        const int u = 4 * it >> per_log2, off = 4 * it & ((1 << per_log2) - 1);
        const int pos = ((__builtin_amdgcn_readfirstlane(chosen.page[u]) << per_log2) + off) * 16;
        if (pos + BN <= limit_min) {
          open = __builtin_amdgcn_readfirstlane(chosen.who[4 * u + wave]) >> token & 1;
          return open ? mx : -INFINITY;
        }
      }
      open = true;
    }
    return mask(it, s) ? lane_max(s) : mx;
  };
  auto reference = [&](bool open) { return CHOSEN && !open ? INFINITY : m * c; };
  // P^T = 2^(S^T c - m c) in bf16 and O^T += V^T P^T.  Probabilities are rounded for the product; the row sum takes them as
  // they are (its logarithm is an output, in fp32).
  auto accumulate = [&](const f32x16 (&s)[2], auto buf_tag, bool open) {
    const float mc = reference(open);
#pragma unroll
    for (int chunk = 0; chunk < 4; ++chunk) {
      bf16x8 va[NV], pb;
#pragma unroll
      for (int i = 0; i < NV; ++i) va[i] = read_v(buf_tag, chunk, i);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = fast_exp2(fmaf(s[chunk >> 1][8 * (chunk & 1) + i], c, -mc));
        l += e;
        pb[i] = static_cast<bf16_t>(e);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[i], pb, o[i], 0, 0, 0);
    }
  };
  constexpr int KPC = NK / 4, NS = 2 * KPC, NA = NV;  // K steps and slots of a phase S, slots of a phase A
  constexpr int SLOTS = 4 * NS + 3 * NA;              // that a copy can go out in
  // Scores of the next tile (K stage kb1) and P V of this one (V stage vb0) together: MFMAs one by one, each with a share of
  // the vector and LDS work behind it, in the order of attend.hip's step: S(g) a quarter of the scores, A(g) the 16 keys of
  // chunk g; the probabilities of chunk g + 1 are formed under A(g) and S(g + 1).  K operands are read under the A before, V
  // operands under the S before: a phase more ahead takes 16 registers, is no faster with bf16 rows (387 and 388 us, 2 x 2048
  // tokens, d = 128), and with 8-bit rows, whose codes come through registers, makes the loop spill (436, 400 us).
  auto step_math = [&](const f32x16 (&s_in)[2], bool open, f32x16 (&s_out)[2], auto kb1, auto vb0, auto&& copy_slot) {
    static_assert(NS == NA && 8 % (NS + NA) == 0, "phases divide the vector work evenly");
    const float mc = reference(open);
    bf16x8 kop[NK][2], vop[4][NV];
    float e[4][8];
    union {
      bf16x8 v;
      bf16x2 h[4];
    } pb[4];
    auto load_k = [&](int ks, int cb) { kop[ks][cb] = read_k(kb1, ks, cb); };
    auto probability = [&](int chunk, int u) {
      e[chunk][u] = fast_exp2(fmaf(s_in[chunk >> 1][8 * (chunk & 1) + u], c, -mc));
      if (u & 1) {
        pb[chunk].h[u >> 1] = bf16x2{static_cast<bf16_t>(e[chunk][u - 1]), static_cast<bf16_t>(e[chunk][u])};
        l += e[chunk][u - 1] + e[chunk][u];
      }
    };
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s_out[cb][r] = 0.f;
    load_k(0, 0);
    load_k(0, 1);
    float mx = -INFINITY;
    int slot = 0;  // compile-time after unrolling
    auto s_slot = [&](int gch, int i, int& done) {
      const int ks = gch * KPC + (i >> 1), cb = i & 1;
      s_out[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[ks][cb], qreg[ks], s_out[cb], 0, 0, 0);
      fence();
      if (gch == 0 && ks + 1 < KPC) load_k(ks + 1, cb);
      vop[gch][i] = read_v(vb0, gch, i);
      copy_slot(slot++);
      const int share = gch == 0 ? 8 / NS : 8 / (NS + NA);
      for (int u = 0; u < share; ++u) probability(gch, done++);
      fence();
    };
    int done = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i) s_slot(0, i, done);
#pragma unroll
    for (int gch = 0; gch < 4; ++gch) {
      done = 0;
#pragma unroll
      for (int d = 0; d < NA; ++d) {
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[gch][d], pb[gch].v, o[d], 0, 0, 0);
        fence();
        if (gch < 3) {
          load_k((gch + 1) * KPC + (d >> 1), d & 1);
          copy_slot(slot++);
#pragma unroll
          for (int u = 0; u < 8 / (NS + NA); ++u) probability(gch + 1, done++);
        } else {  // the new scores are complete: their maxima
#pragma unroll
          for (int r = d * (32 / NA); r < (d + 1) * (32 / NA); ++r) mx = fmaxf(mx, s_out[r >> 4][r & 15]);
          asm volatile("" : "+v"(mx));  // in this slot
        }
        fence();
      }
      if (gch < 3)
#pragma unroll
        for (int i = 0; i < NS; ++i) s_slot(gch + 1, i, done);
    }
    return mx;
  };

  // Step `it`: K(it + 1) and V(it) have landed; V(it + 1) and K(it + 2) go out.  Tile t's K and V lie in stage (t - begin) % 2.
  // `at`: where tile it + 1 lies; tile it + 2 is looked up between the two.
  f32x16 s_a[2], s_b[2];
  TileRows at{};
  // 4-bit rows: codes that are on their way, and the place of the tile whose K they are.
  [[maybe_unused]] Nibbles raw_v, raw_k;
  [[maybe_unused]] Place own{};
  // `math(copy)`: what the wavefront computes in the step; it calls copy(i) for i = 0 .. SLOTS - 1, in order.
  auto step = [&](int it, auto kb1, auto vb0, auto&& math) {
    if constexpr (FP4) {
      // Codes are loaded a step before they are converted, V(it + 2) and K(it + 3) here, and a chunk of 8 columns is converted under a
      // product.  All of a tile's in one place, behind the products of the step that had loaded them, took 382 us instead of 346 for
      // 2 x 2048 tokens over 4096 keys (d = 128), and 80 instead of 68 for whole scales at d = 64 (both with two workgroups to a unit).
      __syncthreads();
      constexpr int CHUNKS = D / 32, GAP = 3, K0 = SLOTS / 2;
      math([&](int i) {
        if (i >= 1 && i < 1 + GAP * CHUNKS && (i - 1) % GAP == 0) store_nibbles(lds[decltype(kb1)::value][1], raw_v, (i - 1) / GAP, One{});
        if (i == 2 + GAP * (CHUNKS - 1)) {
          raw_v = load_v_nibbles(own, it + 2);
          own = locate_own(it + 3);
        }
        if (i >= K0 && i < K0 + GAP * CHUNKS && (i - K0) % GAP == 0) store_nibbles(lds[decltype(vb0)::value][0], raw_k, (i - K0) / GAP, Zero{});
        if (i == K0 + GAP * (CHUNKS - 1) + 1) raw_k = load_nibbles(k_pages, own);
      });
      return;
    }
    wait_vmcnt<0>();
    __syncthreads();
    if constexpr (CODES) {  // V's codes have the first half of the step to arrive, K's the second
      uint4 raw[CPL];
      math([&](int i) {
        if (i == 0)
#pragma unroll
          for (int k = 0; k < CPL; ++k) raw[k] = load_codes(v_pages, at, it + 1, k);
        else if (i == 1)
          at = locate(it + 2);
        else if (i >= SLOTS / 2 && i < SLOTS / 2 + CPL) {
          store_codes(lds[decltype(kb1)::value][1], raw[i - SLOTS / 2], i - SLOTS / 2, One{});
          raw[i - SLOTS / 2] = load_codes(k_pages, at, it + 2, i - SLOTS / 2);
        }
      });
#pragma unroll
      for (int k = 0; k < CPL; ++k) store_codes(lds[decltype(vb0)::value][0], raw[k], k, Zero{});
    } else {
      math([&](int i) {
        if (i < CPT)
          copy_v(at, it + 1, kb1, i);
        else if (i == CPT)
          at = locate(it + 2);
        else if (i >= 2 * CPT && i < 3 * CPT)
          copy_k(at, it + 2, vb0, i - 2 * CPT);
      });
    }
  };
  auto copies_only = [](auto&& copy) {
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) copy(i);
  };
  bool open = true;  // of the scores at hand
  auto pipe_step = [&](int it, auto kb1, auto vb0, f32x16 (&s_in)[2], f32x16 (&s_out)[2]) {
    step(it, kb1, vb0, [&](auto&& copy) {
      const float mx = step_math(s_in, open, s_out, kb1, vb0, copy);
      raise(seen_max(it + 1, s_out, mx, open));
    });
  };
  auto last_step = [&](int it, auto kb1, auto vb0, f32x16 (&s_in)[2]) {
    step(it, kb1, vb0, copies_only);
    accumulate(s_in, vb0, open);
  };
  if (begin < end) {
    const int second = begin + 1 < end ? begin + 1 : begin;
    if constexpr (!FP4) at = locate(begin);
    if constexpr (FP4) {
      own = locate_own(begin);
      raw_k = load_nibbles(k_pages, own);
      raw_v = load_v_nibbles(own, begin);
      own = locate_own(begin + 1);
      const Nibbles next_k = load_nibbles(k_pages, own), next_v = load_v_nibbles(own, begin + 1);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        store_nibbles(lds[0][0], raw_k, k, Zero{});
        store_nibbles(lds[0][1], raw_v, k, One{});
        store_nibbles(lds[1][0], next_k, k, Zero{});
      }
      raw_v = next_v;
      own = locate_own(begin + 2);
      raw_k = load_nibbles(k_pages, own);
    } else if constexpr (CODES) {
      uint4 raw[3][CPL];
#pragma unroll
      for (int k = 0; k < CPL; ++k) {
        raw[0][k] = load_codes(k_pages, at, begin, k);
        raw[1][k] = load_codes(v_pages, at, begin, k);
      }
      at = locate(second);
#pragma unroll
      for (int k = 0; k < CPL; ++k) raw[2][k] = load_codes(k_pages, at, second, k);
#pragma unroll
      for (int k = 0; k < CPL; ++k) {
        store_codes(lds[0][0], raw[0][k], k, Zero{});
        store_codes(lds[0][1], raw[1][k], k, One{});
        store_codes(lds[1][0], raw[2][k], k, Zero{});
      }
    } else {
#pragma unroll
      for (int i = 0; i < CPT; ++i) copy_k(at, begin, Zero{}, i);
#pragma unroll
      for (int i = 0; i < CPT; ++i) copy_v(at, begin, Zero{}, i);
      at = locate(second);
#pragma unroll
      for (int i = 0; i < CPT; ++i) copy_k(at, second, One{}, i);
      wait_vmcnt<2 * CPT>();  // K of the first tile
    }
    __syncthreads();
    if (begin < my_end) {
      scores(s_a, Zero{});
      raise(seen_max(begin, s_a, lane_max(s_a), open));
    }
    // Every wavefront makes all steps (the barriers are shared), those behind its last tile without arithmetic.
    int it = begin;
    for (; it + 2 < my_end; it += 2) {
      pipe_step(it, One{}, Zero{}, s_a, s_b);
      pipe_step(it + 1, Zero{}, One{}, s_b, s_a);
    }
    if (it + 1 < my_end) {
      pipe_step(it, One{}, Zero{}, s_a, s_b);
      last_step(it + 1, Zero{}, One{}, s_b);
      it += 2;
    } else if (it < my_end) {
      last_step(it, One{}, Zero{}, s_a);
      it += 1;
    }
    for (; it < end; ++it)
      if ((it - begin) & 1)
        step(it, Zero{}, One{}, copies_only);
      else
        step(it, One{}, Zero{}, copies_only);
  }

  // Lane (n, hl) holds columns 32 i + 8 (r / 4) + 4 hl + r % 4 of query n.
  l = sum_halves(l);
  const AttendParams& z = arguments();
  const Row out = row_of(z);
  const bool alone = uniform(shared.piece.weight) == 1;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) nan = nan || o[i][r] != o[i][r];
  const unsigned long long nan_lanes = __ballot(nan && out.real);
  if (out.real) {
    const long long token = tl.q0 + out.j, out_row = token * z.c.Hq + out.hq;
    const long long part_row = static_cast<long long>(w) * BM + w_row + n;
    if (hl == 0) {
      if (!alone) {
        z.parts.ml[part_row * 2] = m;
        z.parts.ml[part_row * 2 + 1] = l;
      } else if (z.lse) {
        z.lse[out_row] = natural_lse(m, l, z.sm_scale);
      }
    }
    if (!alone) {
      float* to = z.parts.o + part_row * D + 4 * hl;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f32x4*>(to + 32 * i + 8 * r) = f32x4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
    } else {
      const float f = l > 0.f ? 1.f / l : l;  // nothing seen: zeros; NaN stays
      bf16_t* to = static_cast<bf16_t*>(const_cast<void*>(z.out.data)) + token * z.out.token_stride +
                   out.hq * z.out.head_stride + 4 * hl;
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
  for (unsigned rows = static_cast<unsigned>(nan_lanes | nan_lanes >> 32); rows;) {  // paged_redo.h
    const int r = __builtin_ctz(rows);
    rows &= rows - 1;
    wait_vmcnt<0>();  // the row's outputs from above, which other lanes have written, come first
    __threadfence_block();
    const int j = __builtin_amdgcn_readlane(out.j, r), hq = __builtin_amdgcn_readlane(out.hq, r);
    const float m_row = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), r));
    const float l_row = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, l), r));
    const bool lost = CHOSEN && l_row != l_row;  // a score that is not finite, of a page that other rows have chosen or this one
    const long long part_row = static_cast<long long>(w) * BM + w_row + r;
    float* const parts_row = z.parts.o + part_row * D;  // the part's, or not used
    bf16_t* const out_row = static_cast<bf16_t*>(const_cast<void*>(z.out.data)) + (tl.q0 + j) * z.out.token_stride + hq * z.out.head_stride;
    const float l_seen = redo_row<bf16_t, F, D, CHOSEN>(
        z, tl.q0 + j, hq, visible_keys(z.c, tl, j), tl.len, 4 * begin, 4 * end, lost,
        [&](int g) {
          if constexpr (CHOSEN) {
            const int u = g >> per_log2, off = g & ((1 << per_log2) - 1);
            if (u >= n_pages || !(chosen.who[4 * u + wave] >> (j - w_first) & 1)) return RedoGranule{0, 0, false};
            return RedoGranule{(static_cast<long long>(__builtin_amdgcn_readfirstlane(chosen.granule[u])) + off) * 16,
                               ((__builtin_amdgcn_readfirstlane(chosen.page[u]) << per_log2) + off) * 16, true};
          }
          const TileRows rows_at = locate(g >> 2);
          const int from = g & 2 ? (g & 1 ? rows_at.granule[3] : rows_at.granule[2]) : (g & 1 ? rows_at.granule[1] : rows_at.granule[0]);
          return RedoGranule{static_cast<long long>(from) * 16, 16 * g, true};
        },
        [&](float score) { return fast_exp2((score - m_row) * c); },
        [&](int col) { return alone ? static_cast<float>(out_row[col]) : parts_row[col]; },
        [&](int col, float x, float sum) {
          const float l_all = lost ? sum : l_row;
          if (!alone)
            parts_row[col] = x;
          else
            out_row[col] = static_cast<bf16_t>(x * (l_all > 0.f ? 1.f / l_all : l_all));
        });
    if (lost && lane == 0) {
      if (!alone)
        z.parts.ml[part_row * 2 + 1] = l_seen;
      else if (z.lse)
        z.lse[(tl.q0 + j) * static_cast<long long>(z.c.Hq) + hq] = natural_lse(m_row, l_seen, z.sm_scale);
    }
  }
}

template <int D, Format F, bool CHOSEN>
hipError_t launch(const AttendParams& p, const AttendParams& few, int kv_format, hipStream_t stream) {
  static_assert(FEW_WAVES * stage_bytes(D) + FEW_SHARED <= 4 * BN * 2 * D + kUnionAt, "the workgroups of few rows have room");
  // With chosen pages as well: walk_lds_bytes() is for the union of no more tokens, of which each page takes 8 bytes instead of 24.
  const size_t lds = 4 * BN * 2 * D + kUnionAt + (CHOSEN ? many_union_bytes(p.c.G, p.c.max_pages, p.top) : 0);
  static std::atomic<unsigned long long> allowed{0};
  if (lds > 64 * 1024)
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(&paged_attend_long_kernel<D, F, CHOSEN>), MANY_LDS, allowed)) return e;
  const FewRows place = place_of_few(p.c.batch, CHOSEN, lds, row_bytes<bf16_t, F>(D));
  AttendParams along = few;
  if (place == FewRows::APART) along.parts.grid = 0;
  hipLaunchKernelGGL((paged_attend_long_kernel<D, F, CHOSEN>), dim3(p.parts.grid + along.parts.grid), dim3(256), lds, stream, p, along,
                     place == FewRows::IN_FRONT ? 0 : p.parts.grid);
  if (hipError_t e = hipGetLastError()) return e;
  return place == FewRows::APART ? launch_paged_attend_bf16(few, D, kv_format, stream) : hipSuccess;
}

}  // namespace

hipError_t launch_paged_attend_long(const PagedAttendParams& p, const PagedAttendParams& few, int d, int kv_format, hipStream_t stream) {
  static_assert(4 * BN * 2 * 128 + kUnionAt + MANY_UNION_BYTES <= MANY_LDS, "the largest union that plan_launches() sends here fits");
  auto run = [&](auto d_tag, auto chosen) {
    constexpr int D = decltype(d_tag)::value;
    constexpr bool CHOSEN = decltype(chosen)::value;
    return kv_format == HEATKV_KV_FP4_E2M1   ? launch<D, E2M1, CHOSEN>(p, few, kv_format, stream)
           : kv_format == HEATKV_KV_FP8_E4M3 ? launch<D, E4M3, CHOSEN>(p, few, kv_format, stream)
                                             : launch<D, NATIVE, CHOSEN>(p, few, kv_format, stream);
  };
  using D128 = std::integral_constant<int, 128>;
  using D64 = std::integral_constant<int, 64>;
  if (p.selected) return d == 128 ? run(D128{}, std::true_type{}) : run(D64{}, std::true_type{});
  return d == 128 ? run(D128{}, std::false_type{}) : run(D64{}, std::false_type{});
}

}  // namespace heatkv
