// extern "C" entry points of the paged cache: argument checks and the hand-off to the kernel launchers.
#include <climits>
#include <cmath>
#include <cstdint>
#include <string>
#include <utility>

#include <hip/hip_runtime.h>

#include "heatkv.h"
#include "kernels.h"
#include "paged.h"
#include "paged_schedule.h"
#include "paged_rules.h"
#include "plan.h"

using heatkv::fail;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 22;      // rows of the token tensors
constexpr int64_t kMaxTokenHeads = int64_t(1) << 23;  // times kv heads
constexpr int64_t kMaxPositions = int64_t(1) << 30;   // keys of a request, rows of the cache per kv head
constexpr int kMaxGroup = 16, kMaxTop = 512, kMaxSelectPages = 32768;

int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

int check_shape(const heatkv_paged_shape* s) {
  if (!s) return fail(HEATKV_EINVAL, "paged shape is null");
  if (s->kv_heads < 1 || s->q_heads < 1) return fail(HEATKV_EINVAL, "q_heads and kv_heads must be >= 1");
  if (s->q_heads % s->kv_heads != 0) return fail(HEATKV_EINVAL, "q_heads must be a multiple of kv_heads");
  if (s->q_heads / s->kv_heads > kMaxGroup) return fail(HEATKV_EINVAL, "more than 16 query heads share a kv head");
  if (s->kv_heads > 1024) return fail(HEATKV_EINVAL, "more than 1024 kv heads");
  if (s->d != 64 && s->d != 128) return fail(HEATKV_EINVAL, "head dimension must be 64 or 128");
  if (s->dtype != HEATKV_F32 && s->dtype != HEATKV_BF16) return fail(HEATKV_EINVAL, "unknown dtype");
  if (s->kv_format != HEATKV_KV_NATIVE && s->kv_format != HEATKV_KV_FP8_E4M3 && s->kv_format != HEATKV_KV_FP4_E2M1)
    return fail(HEATKV_EINVAL, "unknown cache storage format");
  if (s->kv_format == HEATKV_KV_FP8_E4M3 && s->dtype != HEATKV_BF16)
    return fail(HEATKV_EINVAL, "HEATKV_KV_FP8_E4M3 needs a bf16 shape");
  if (s->kv_format == HEATKV_KV_FP4_E2M1 && s->dtype != HEATKV_BF16)
    return fail(HEATKV_EINVAL, "HEATKV_KV_FP4_E2M1 needs a bf16 shape");
  if (s->page_size < 16 || s->page_size > 256 || (s->page_size & (s->page_size - 1)) != 0)
    return fail(HEATKV_EINVAL, "page_size must be 16, 32, 64, 128 or 256");
  if (s->batch < 1 || s->batch > heatkv::paged::MAX_BATCH) return fail(HEATKV_EINVAL, "batch must be in [1, 4096]");
  if (s->num_pages < 1 || int64_t(s->num_pages) * s->page_size > kMaxPositions)
    return fail(HEATKV_EINVAL, "num_pages must be >= 1, and num_pages * page_size at most 2^30");
  if (int64_t(s->num_pages) * s->page_size * s->kv_heads > int64_t(1) << 34)
    return fail(HEATKV_EINVAL, "num_pages * page_size * kv_heads must be at most 2^34");
  if (s->max_pages < 1 || int64_t(s->max_pages) * s->page_size > kMaxPositions)
    return fail(HEATKV_EINVAL, "max_pages must be >= 1, and max_pages * page_size at most 2^30");
  return HEATKV_OK;
}

int check_tokens(int64_t tokens) {
  if (tokens < 0 || tokens > kMaxTokens) return fail(HEATKV_EINVAL, "tokens must be in [0, 2^22]");
  return HEATKV_OK;
}

// Of calls whose work is by tokens and kv heads: a launch has less than 2^32 lanes, up to 256 for each of them.
int check_tokens(const heatkv_paged_shape* s, int64_t tokens) {
  if (int rc = check_tokens(tokens)) return rc;
  if (tokens * s->kv_heads > kMaxTokenHeads) return fail(HEATKV_EINVAL, "tokens * kv_heads must be at most 2^23");
  return HEATKV_OK;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Rows of a token tensor: read and written 16 bytes at a time.
int check_rows(const heatkv_paged_shape* s, const heatkv_rows& r, const char* name) {
  if (!r.data) return fail(HEATKV_EINVAL, std::string(name) + " is null");
  const int64_t elem = s->dtype == HEATKV_BF16 ? 2 : 4;
  if (!aligned(r.data, 16) || r.token_stride * elem % 16 != 0 || r.head_stride * elem % 16 != 0)
    return fail(HEATKV_EINVAL, std::string(name) + ": address and strides must be multiples of 16 bytes");
  return HEATKV_OK;
}

// Rows that are written: no two of them share an element.
int check_apart(const heatkv_paged_shape* s, int64_t tokens, int64_t heads, const heatkv_rows& r, const char* name) {
  const int64_t t = r.token_stride, h = r.head_stride, d = s->d;
  const bool apart = (tokens == 1 || t >= d) && (heads == 1 || h >= d) &&
                     (tokens == 1 || heads == 1 || t >= (heads - 1) * h + d || h >= (tokens - 1) * t + d);
  return apart ? HEATKV_OK : fail(HEATKV_EINVAL, std::string(name) + ": rows overlap one another");
}

int check_cache(const void* k_pages, const void* v_pages) {
  if (!k_pages || !v_pages) return fail(HEATKV_EINVAL, "null page pointer");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return fail(HEATKV_EINVAL, "pages must be 16-byte aligned");
  return HEATKV_OK;
}

int check_bounds(const int8_t* bounds, const float* bound_scales) {
  if ((bounds == nullptr) != (bound_scales == nullptr)) return fail(HEATKV_EINVAL, "bounds and bound_scales go together");
  if (bounds && (!aligned(bounds, 16) || !aligned(bound_scales, 4)))
    return fail(HEATKV_EINVAL, "bounds must be 16-byte aligned, bound_scales 4-byte");
  return HEATKV_OK;
}

int check_ints(std::initializer_list<const void*> arrays) {
  for (const void* a : arrays) {
    if (!a) return fail(HEATKV_EINVAL, "null integer array");
    if (!aligned(a, 4)) return fail(HEATKV_EINVAL, "integer arrays must be 4-byte aligned");
  }
  return HEATKV_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// One array of a call: the addresses of its first byte and of the one behind its last.
struct Span {
  const char* name;
  uintptr_t first, end;
  bool written;
};
constexpr bool READ = false, WRITTEN = true;
Span span_of(const char* name, const void* p, size_t bytes, bool written) {
  const auto first = reinterpret_cast<uintptr_t>(p);
  return {name, first, first + (p ? bytes : 0), written};
}
Span span_of(const char* name, const heatkv_paged_shape* s, const heatkv_rows& r, int64_t tokens, int64_t heads, bool written) {
  const int elem = s->dtype == HEATKV_BF16 ? 2 : 4;
  const __int128 t = static_cast<__int128>(r.token_stride) * (tokens - 1), h = static_cast<__int128>(r.head_stride) * (heads - 1);
  const auto at = static_cast<__int128>(reinterpret_cast<uintptr_t>(r.data));
  const __int128 first = at + (std::min<__int128>(t, 0) + std::min<__int128>(h, 0)) * elem;
  const __int128 end = at + (std::max<__int128>(t, 0) + std::max<__int128>(h, 0) + s->d) * elem;
  return {name, static_cast<uintptr_t>(std::max<__int128>(first, 0)), static_cast<uintptr_t>(std::min<__int128>(end, UINTPTR_MAX)), written};
}
bool meet(const Span& a, const Span& b) { return a.first < b.end && b.first < a.end && a.first < a.end && b.first < b.end; }
// Workgroups run in any order: what a call writes, it neither reads through another argument nor writes twice.  Arrays that are
// written come first.
int check_disjoint(const Span* first, const Span* end) {
  for (const Span* a = first; a != end && a->written; ++a)
    for (const Span* b = a + 1; b != end; ++b)
      if (meet(*a, *b)) return fail(HEATKV_EINVAL, std::string(a->name) + " overlaps " + b->name);
  return HEATKV_OK;
}
int check_disjoint(std::initializer_list<Span> arrays) { return check_disjoint(arrays.begin(), arrays.end()); }
// Whether rows that are written (check_apart() holds) have an element in common with others.  Where their ranges overlap: not if
// they are slices of one tensor, beside each other; rows that go by different strides are taken to meet.
bool rows_meet(const heatkv_paged_shape* s, const heatkv_rows& out, const heatkv_rows& in, int64_t tokens, int64_t heads) {
  if (!meet(span_of("", s, out, tokens, heads, WRITTEN), span_of("", s, in, tokens, heads, READ))) return false;
  if ((tokens > 1 && out.token_stride != in.token_stride) || (heads > 1 && out.head_stride != in.head_stride)) return true;
  struct Axis {
    __int128 stride, count;
  };
  Axis outer{out.token_stride, tokens}, inner{out.head_stride, heads};
  if (tokens == 1 || (heads > 1 && inner.stride > outer.stride)) std::swap(outer, inner);
  for (Axis* x : {&outer, &inner})
    if (x->count == 1) x->stride = static_cast<__int128>(1) << 80;  // not used
  const __int128 bytes = static_cast<__int128>(reinterpret_cast<uintptr_t>(in.data)) - reinterpret_cast<uintptr_t>(out.data);
  const __int128 off = bytes / (s->dtype == HEATKV_BF16 ? 2 : 4);
  auto floor = [](__int128 n, __int128 d) { return n / d - (n % d < 0); };
  // Steps of the outer axis between two rows that meet (few: the inner axis lies within one), then the nearest of the inner one.
  const __int128 reach = (inner.count - 1) * inner.stride + s->d;
  const __int128 last = std::min(outer.count - 1, floor(off + reach, outer.stride));
  for (__int128 i = std::max(1 - outer.count, floor(off - reach, outer.stride)); i <= last; ++i) {
    const __int128 rest = off - i * outer.stride;
    __int128 j = floor(rest, inner.stride);
    for (int near = 0; near < 2; ++near, ++j) {
      const __int128 apart = rest - j * inner.stride;
      if (j < inner.count && -j < inner.count && apart < s->d && -apart < s->d) return true;
    }
  }
  return false;
}
size_t pages_bytes(const heatkv_paged_shape* s) {
  const int row = s->kv_format == HEATKV_KV_FP4_E2M1   ? s->d / 2 + s->d / 32
                  : s->kv_format == HEATKV_KV_FP8_E4M3 ? s->d
                                                       : s->d * (s->dtype == HEATKV_F32 ? 4 : 2);
  return size_t(s->num_pages) * s->page_size * s->kv_heads * row;
}
size_t table_bytes(const heatkv_paged_shape* s) { return size_t(s->batch) * s->max_pages * 4; }

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? HEATKV_OK : fail(HEATKV_EHIP, std::string(what) + " launch: " + hipGetErrorString(e));
}

heatkv::paged::Cache cache_of(const heatkv_paged_shape* s, int64_t tokens, const int32_t* table, const int32_t* q_start,
                              const int32_t* lens, int causal) {
  heatkv::paged::Cache c{};
  c.H = s->kv_heads;
  c.G = s->q_heads / s->kv_heads;
  c.Hq = s->q_heads;
  c.page_log2 = log2_of(s->page_size);
  c.num_pages = s->num_pages;
  c.batch = s->batch;
  c.max_pages = s->max_pages;
  c.tokens = int(tokens);
  c.div_G = heatkv::paged::reciprocal(unsigned(c.G));
  c.causal = causal ? 1 : 0;
  c.table = table;
  c.q_start = q_start;
  c.lens = lens;
  return c;
}

// Workspace: the parts of cut segments, of the few-row launch and of the long one, each array from a multiple of 256 bytes on.
struct PartArrays {
  size_t o = 0, ml = 0, borders = 0;
};
struct Workspace {
  PartArrays few, many;
  size_t total = 0;
};
Workspace workspace_of(const heatkv_paged_shape* s, const heatkv::paged::Plan& plan) {
  Workspace w;
  auto take = [&](size_t n) {
    const size_t at = w.total;
    w.total += (n + 255) / 256 * 256;
    return at;
  };
  auto arrays = [&](PartArrays& a, const heatkv::paged::Launch& l, int rows) {
    if (!l.parts) return;
    a.o = take(size_t(l.parts) * rows * s->d * 4);
    a.ml = take(size_t(l.parts) * rows * 8);
    a.borders = take(size_t(l.grid) * sizeof(heatkv::paged::Border));
  };
  arrays(w.few, plan.few, 16);
  arrays(w.many, plan.many, 128);
  return w;
}

heatkv::paged::Plan plan_of(const heatkv_paged_shape* s, int64_t tokens, int top) {
  return heatkv::paged::plan_launches(s->dtype == HEATKV_BF16, s->batch, s->kv_heads, s->q_heads / s->kv_heads, tokens,
                                      s->max_pages, s->page_size, top);
}

int attend(const heatkv_paged_shape* s, int64_t tokens, heatkv_rows q, const void* k_pages, const void* v_pages,
           const int32_t* table, const int32_t* q_start, const int32_t* lens, const int32_t* selected, int top, float sm_scale,
           int causal, heatkv_rows out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(s, tokens);
  if (rc) return rc;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return fail(HEATKV_EINVAL, "sm_scale must be positive and finite");
  if (tokens == 0) return HEATKV_OK;
  if (!rc) rc = check_rows(s, q, "q");
  if (!rc) rc = check_rows(s, out, "out");
  if (!rc) rc = check_apart(s, tokens, s->q_heads, out, "out");
  if (!rc) rc = check_cache(k_pages, v_pages);
  if (!rc) rc = check_ints({table, q_start, lens});
  if (rc) return rc;
  if (lse && !aligned(lse, 4)) return fail(HEATKV_EINVAL, "lse must be 4-byte aligned");
  const auto plan = plan_of(s, tokens, top);
  const Workspace w = workspace_of(s, plan);
  if (w.total > 0) {
    if (!ws || ws_bytes < w.total) return fail(HEATKV_EINVAL, "paged attention workspace too small");
    if (!aligned(ws, 16)) return fail(HEATKV_EINVAL, "workspace must be 16-byte aligned");
  }
  const size_t requests = size_t(s->batch) * 4;
  const Span lse_span = span_of("lse", lse, size_t(tokens) * s->q_heads * 4, WRITTEN), ws_span = span_of("ws", ws, w.total, WRITTEN);
  rc = check_disjoint({span_of("out", s, out, tokens, s->q_heads, WRITTEN), lse_span, ws_span,
                       span_of("k_pages", k_pages, pages_bytes(s), READ), span_of("v_pages", v_pages, pages_bytes(s), READ),
                       span_of("table", table, table_bytes(s), READ), span_of("q_start", q_start, requests + 4, READ),
                       span_of("lens", lens, requests, READ),
                       span_of("selected", selected, size_t(tokens) * s->kv_heads * top * 4, READ)});
  if (!rc) rc = check_disjoint({lse_span, ws_span, span_of("q", s, q, tokens, s->q_heads, READ)});
  if (rc) return rc;
  if (rows_meet(s, out, q, tokens, s->q_heads)) return fail(HEATKV_EINVAL, "out overlaps q");
  heatkv::paged::AttendParams p{};
  p.c = cache_of(s, tokens, table, q_start, lens, causal);
  p.q = {q.data, q.token_stride, q.head_stride};
  p.out = {out.data, out.token_stride, out.head_stride};
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.selected = selected;
  p.top = top;
  p.sm_scale = sm_scale;
  p.lse = lse;
  const auto hip_stream = static_cast<hipStream_t>(stream);
  // The arguments of one of the two kernels.
  auto arguments = [&](const heatkv::paged::Launch& l, const PartArrays& a) {
    heatkv::paged::AttendParams x = p;
    if (!l.workgroups) return x;  // no grid
    if (l.parts) {
      x.parts.o = reinterpret_cast<float*>(static_cast<char*>(ws) + a.o);
      x.parts.ml = reinterpret_cast<float*>(static_cast<char*>(ws) + a.ml);
      x.parts.borders = reinterpret_cast<heatkv::paged::Border*>(static_cast<char*>(ws) + a.borders);
    }
    x.parts.grid = int(l.grid);
    x.workgroups = l.workgroups;
    x.least_weight = l.least_steps * heatkv::paged::STEP_WEIGHT;
    x.cut_from = l.parts ? x.least_weight : INT_MAX;
    x.least_rows = l.least_rows;
    x.most_rows = l.most_rows;
    x.whole_from = l.whole_from;
    return x;
  };
  heatkv::paged::AttendParams many = arguments(plan.many, w.many), few = arguments(plan.few, w.few);
  hipError_t e = many.parts.grid > 0      ? heatkv::launch_paged_attend_long(many, few, s->d, s->kv_format, hip_stream)
                 : s->dtype == HEATKV_F32 ? heatkv::launch_paged_attend_f32(few, s->d, hip_stream)
                                          : heatkv::launch_paged_attend_bf16(few, s->d, s->kv_format, hip_stream);
  // The join looks at the workgroups that may have parts.
  many.parts.grid = many.parts.grid > 0 ? heatkv::paged::join_workgroups(plan.many) : 0;
  few.parts.grid = heatkv::paged::join_workgroups(plan.few);
  if (e == hipSuccess && few.parts.grid + many.parts.grid > 0)
    e = heatkv::launch_paged_join(few, few.parts, many.parts, s->dtype, s->d, hip_stream);
  return launched(e, "paged_attend");
}

// Workspace of the calls on shared pages, each array from a multiple of 256 bytes on.  A workgroup of compact looks at `tile` tokens
// of a row of the table: few enough that 256 of them are a row.
struct TablesWorkspace {
  size_t state, next, gone, per_row[5], counts, drops, total = 0;
  int tile = 4096, tiles;
};
TablesWorkspace tables_workspace_of(const heatkv_paged_shape* s) {
  TablesWorkspace w;
  auto take = [&](size_t n) {
    const size_t at = w.total;
    w.total += (n + 255) / 256 * 256;
    return at;
  };
  const int64_t longest = int64_t(s->max_pages) * s->page_size;
  while ((longest + w.tile - 1) / w.tile > 256) w.tile *= 2;
  w.tiles = int((longest + w.tile - 1) / w.tile);
  w.state = take(64);
  w.next = take(size_t(s->batch) * 4);
  w.gone = take((size_t(s->num_pages) + 31) / 32 * 4);
  for (size_t& at : w.per_row) at = take((size_t(s->batch) + 1) * 4);
  w.counts = take(size_t(s->batch) * w.tiles * 4);
  w.drops = take(size_t(s->batch) * w.tiles * 4);
  return w;
}

// What the calls on shared pages have in common: their arrays, and how they are checked.
struct Tables {
  const heatkv_paged_shape* s;
  const int32_t* lens;
  int32_t *lens_out, *holders, *free_ring;
  const int32_t* free_span;
  int32_t *free_span_out, *table, *status;
  void* ws;
  size_t ws_bytes;
  TablesWorkspace w{};

  int check() {
    if (int rc = check_shape(s)) return rc;
    if (int64_t(s->batch) * s->max_pages > int64_t(1) << 30) return fail(HEATKV_EINVAL, "batch * max_pages must be at most 2^30");
    if (int rc = check_ints({lens, lens_out, holders, free_ring, free_span, free_span_out, table, status})) return rc;
    w = tables_workspace_of(s);
    if (!ws || ws_bytes < w.total) return fail(HEATKV_EINVAL, "tables workspace too small");
    if (!aligned(ws, 16)) return fail(HEATKV_EINVAL, "workspace must be 16-byte aligned");
    return HEATKV_OK;
  }
  // `written`, `read`: the call's own arrays.
  int check_apart_from(std::initializer_list<Span> written, std::initializer_list<Span> read) const {
    const size_t row = size_t(s->batch) * 4;
    if (lens_out != lens && overlap(lens_out, row, lens, row)) return fail(HEATKV_EINVAL, "lens_out overlaps lens in part");
    if (free_span_out != free_span && overlap(free_span_out, 8, free_span, 8))
      return fail(HEATKV_EINVAL, "free_span_out overlaps free_span in part");
    Span all[24] = {span_of("lens_out", lens_out, row, WRITTEN), span_of("free_span_out", free_span_out, 8, WRITTEN),
                    span_of("holders", holders, size_t(s->num_pages) * 4, WRITTEN),
                    span_of("free_ring", free_ring, size_t(s->num_pages) * 4, WRITTEN),
                    span_of("table", table, table_bytes(s), WRITTEN), span_of("status", status, 4, WRITTEN),
                    span_of("ws", ws, w.total, WRITTEN)};
    int n = 7;
    for (const Span& x : written) all[n++] = x;
    all[n++] = span_of("lens", lens, lens_out == lens ? 0 : row, READ);
    all[n++] = span_of("free_span", free_span, free_span_out == free_span ? 0 : 8, READ);
    for (const Span& x : read) all[n++] = x;
    return check_disjoint(all, all + n);
  }
  template <class X>
  X* at(size_t offset) const { return reinterpret_cast<X*>(static_cast<char*>(ws) + offset); }
  heatkv::TableArgs args() const {
    heatkv::TableArgs t{};
    t.batch = s->batch;
    t.num_pages = s->num_pages;
    t.max_pages = s->max_pages;
    t.page_log2 = log2_of(s->page_size);
    t.lens = lens;
    t.span = free_span;
    t.lens_out = lens_out;
    t.span_out = free_span_out;
    t.holders = holders;
    t.ring = free_ring;
    t.table = table;
    t.status = status;
    t.state = at<int32_t>(w.state);
    t.next = at<int32_t>(w.next);
    t.gone = at<uint32_t>(w.gone);
    return t;
  }
};

}  // namespace

extern "C" {

int heatkv_paged_assign(const heatkv_paged_shape* s, const int32_t* keep, const int32_t* new_tokens, const int32_t* lens,
                        int32_t* lens_out, int32_t* free_ring, const int32_t* free_span, int32_t* free_span_out, int32_t* table,
                        int32_t* q_start, int32_t* slots, int64_t max_tokens, int32_t* status, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(max_tokens);
  if (!rc) rc = check_ints({keep, new_tokens, lens, lens_out, free_ring, free_span, free_span_out, table, q_start, status});
  if (!rc && max_tokens > 0) rc = check_ints({slots});
  if (rc) return rc;
  const size_t row = size_t(s->batch) * 4;
  if (lens_out != lens && overlap(lens_out, row, lens, row)) return fail(HEATKV_EINVAL, "lens_out overlaps lens in part");
  if (free_span_out != free_span && overlap(free_span_out, 8, free_span, 8))
    return fail(HEATKV_EINVAL, "free_span_out overlaps free_span in part");
  if (overlap(lens_out, row, keep, row) || overlap(lens_out, row, new_tokens, row))
    return fail(HEATKV_EINVAL, "keep and new_tokens must not overlap lens_out");
  rc = check_disjoint({span_of("lens_out", lens_out, row, WRITTEN), span_of("free_ring", free_ring, size_t(s->num_pages) * 4, WRITTEN),
                       span_of("free_span_out", free_span_out, 8, WRITTEN), span_of("table", table, table_bytes(s), WRITTEN),
                       span_of("q_start", q_start, row + 4, WRITTEN), span_of("slots", slots, size_t(max_tokens) * 4, WRITTEN),
                       span_of("status", status, 4, WRITTEN), span_of("keep", keep, row, READ),
                       span_of("new_tokens", new_tokens, row, READ), span_of("lens", lens, lens_out == lens ? 0 : row, READ),
                       span_of("free_span", free_span, free_span_out == free_span ? 0 : 8, READ)});
  if (rc) return rc;
  heatkv::AssignArgs a{};
  a.batch = s->batch;
  a.num_pages = s->num_pages;
  a.max_pages = s->max_pages;
  a.page_log2 = log2_of(s->page_size);
  a.max_tokens = max_tokens;
  a.keep = keep;
  a.new_tokens = new_tokens;
  a.lens = lens;
  a.span = free_span;
  a.lens_out = lens_out;
  a.span_out = free_span_out;
  a.ring = free_ring;
  a.table = table;
  a.q_start = q_start;
  a.slots = slots;
  a.status = status;
  return launched(heatkv::launch_paged_assign(a, static_cast<hipStream_t>(stream)), "paged_assign");
}

int heatkv_paged_append(const heatkv_paged_shape* s, const int32_t* slots, int64_t tokens, heatkv_rows k_new, heatkv_rows v_new,
                        void* k_pages, void* v_pages, int8_t* bounds, float* bound_scales, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(s, tokens);
  if (rc || tokens == 0) return rc;
  rc = check_ints({slots});
  if (!rc) rc = check_rows(s, k_new, "k_new");
  if (!rc) rc = check_rows(s, v_new, "v_new");
  if (!rc) rc = check_cache(k_pages, v_pages);
  if (rc) return rc;
  if ((rc = check_bounds(bounds, bound_scales))) return rc;
  const size_t pages_heads = size_t(s->num_pages) * s->kv_heads;
  const Span bounds_span = span_of("bounds", bounds, pages_heads * 2 * s->d, WRITTEN),
             scales_span = span_of("bound_scales", bound_scales, pages_heads * 4, WRITTEN);
  rc = check_disjoint({span_of("k_pages", k_pages, pages_bytes(s), WRITTEN), span_of("v_pages", v_pages, pages_bytes(s), WRITTEN),
                       bounds_span, scales_span, span_of("slots", slots, size_t(tokens) * 4, READ)});
  // The new rows may be other rows of the pages: that is how a page is copied.
  if (!rc)
    rc = check_disjoint({bounds_span, scales_span, span_of("k_new", s, k_new, tokens, s->kv_heads, READ),
                         span_of("v_new", s, v_new, tokens, s->kv_heads, READ)});
  if (rc) return rc;
  heatkv::PagedAppendArgs a{};
  a.dtype = s->dtype;
  a.d = s->d;
  a.H = s->kv_heads;
  a.page_log2 = log2_of(s->page_size);
  a.num_pages = s->num_pages;
  a.kv_format = s->kv_format;
  a.tokens = tokens;
  a.slots = slots;
  a.k_new = k_new.data;
  a.v_new = v_new.data;
  a.k_token_stride = k_new.token_stride;
  a.k_head_stride = k_new.head_stride;
  a.v_token_stride = v_new.token_stride;
  a.v_head_stride = v_new.head_stride;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.bounds = bounds;
  a.bound_scales = bound_scales;
  return launched(heatkv::launch_paged_append(a, static_cast<hipStream_t>(stream)), "paged_append");
}

size_t heatkv_paged_attend_workspace_bytes(const heatkv_paged_shape* s, int64_t tokens, int top) {
  if (check_shape(s) || check_tokens(s, tokens)) return 0;
  if (top < 0 || top > kMaxTop) return 0;
  return workspace_of(s, plan_of(s, tokens, top)).total;
}

int heatkv_paged_attend(const heatkv_paged_shape* s, int64_t tokens, heatkv_rows q, const void* k_pages, const void* v_pages,
                        const int32_t* table, const int32_t* q_start, const int32_t* lens, float sm_scale, int causal,
                        heatkv_rows out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attend(s, tokens, q, k_pages, v_pages, table, q_start, lens, nullptr, 0, sm_scale, causal, out, lse, ws, ws_bytes,
                stream);
}

int heatkv_paged_select(const heatkv_paged_shape* s, int64_t tokens, heatkv_rows q, const int8_t* bounds,
                        const float* bound_scales, const int32_t* table, const int32_t* q_start, const int32_t* lens, int first,
                        int last, int top, int causal, int32_t* selected, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(s, tokens);
  if (rc) return rc;
  if (top < 1 || top > kMaxTop) return fail(HEATKV_EINVAL, "top must be in [1, 512]");
  if (first < 0 || last < 1 || int64_t(first) + last > top)
    return fail(HEATKV_EINVAL, "first >= 0, last >= 1 and first + last <= top are needed");
  if (s->max_pages > kMaxSelectPages) return fail(HEATKV_EINVAL, "the choice of pages takes requests of up to 32768 pages");
  if (tokens == 0) return HEATKV_OK;
  rc = check_rows(s, q, "q");
  if (!rc) rc = check_ints({table, q_start, lens, selected, bound_scales});
  if (rc) return rc;
  if (!bounds || !aligned(bounds, 16)) return fail(HEATKV_EINVAL, "bounds must be 16-byte aligned and not null");
  const size_t pages_heads = size_t(s->num_pages) * s->kv_heads, requests = size_t(s->batch) * 4;
  rc = check_disjoint({span_of("selected", selected, size_t(tokens) * s->kv_heads * top * 4, WRITTEN),
                       span_of("q", s, q, tokens, s->q_heads, READ), span_of("bounds", bounds, pages_heads * 2 * s->d, READ),
                       span_of("bound_scales", bound_scales, pages_heads * 4, READ), span_of("table", table, table_bytes(s), READ),
                       span_of("q_start", q_start, requests + 4, READ), span_of("lens", lens, requests, READ)});
  if (rc) return rc;
  heatkv::PagedSelectParams p{};
  p.c = cache_of(s, tokens, table, q_start, lens, causal);
  p.tokens_as_rows = p.c;
  p.tokens_as_rows.G = 1;
  p.tokens_as_rows.div_G = 0;
  p.q = {q.data, q.token_stride, q.head_stride};
  p.bounds = bounds;
  p.bound_scales = bound_scales;
  p.first = first;
  p.last = last;
  p.top = top;
  p.selected = selected;
  return launched(heatkv::launch_paged_select(p, s->dtype, s->d, static_cast<hipStream_t>(stream)), "paged_select");
}

int heatkv_paged_attend_selected(const heatkv_paged_shape* s, int64_t tokens, heatkv_rows q, const void* k_pages,
                                 const void* v_pages, const int32_t* table, const int32_t* q_start, const int32_t* lens,
                                 const int32_t* selected, int top, float sm_scale, int causal, heatkv_rows out, float* lse,
                                 void* ws, size_t ws_bytes, void* stream) {
  int rc = check_shape(s);
  if (rc) return rc;
  if (top < 1 || top > kMaxTop) return fail(HEATKV_EINVAL, "top must be in [1, 512]");
  if (s->max_pages > kMaxSelectPages) return fail(HEATKV_EINVAL, "chosen pages: requests of up to 32768 pages");
  if (tokens != 0 && (rc = check_ints({selected}))) return rc;
  return attend(s, tokens, q, k_pages, v_pages, table, q_start, lens, selected, top, sm_scale, causal, out, lse, ws, ws_bytes,
                stream);
}

int heatkv_paged_move(const heatkv_paged_shape* s, const int32_t* move_from, const int32_t* move_to, int64_t rows, void* k_pages,
                      void* v_pages, int8_t* bounds, float* bound_scales, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(s, rows);
  if (rc || rows == 0) return rc;
  rc = check_ints({move_from, move_to});
  if (!rc) rc = check_cache(k_pages, v_pages);
  if (!rc) rc = check_bounds(bounds, bound_scales);
  if (rc) return rc;
  const size_t pages_heads = size_t(s->num_pages) * s->kv_heads, list = size_t(rows) * 4;
  rc = check_disjoint({span_of("k_pages", k_pages, pages_bytes(s), WRITTEN), span_of("v_pages", v_pages, pages_bytes(s), WRITTEN),
                       span_of("bounds", bounds, pages_heads * 2 * s->d, WRITTEN),
                       span_of("bound_scales", bound_scales, pages_heads * 4, WRITTEN), span_of("move_from", move_from, list, READ),
                       span_of("move_to", move_to, list, READ)});
  if (rc) return rc;
  heatkv::PagedAppendArgs a{};
  a.dtype = s->dtype;
  a.d = s->d;
  a.H = s->kv_heads;
  a.page_log2 = log2_of(s->page_size);
  a.num_pages = s->num_pages;
  a.kv_format = s->kv_format;
  a.tokens = rows;
  a.slots = move_to;
  a.from = move_from;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.bounds = bounds;
  a.bound_scales = bound_scales;
  return launched(heatkv::launch_paged_append(a, static_cast<hipStream_t>(stream)), "paged_move");
}

int heatkv_paged_read(const heatkv_paged_shape* s, const int32_t* slots, int64_t tokens, const void* k_pages, const void* v_pages,
                      heatkv_rows k_out, heatkv_rows v_out, void* stream) {
  int rc = check_shape(s);
  if (!rc) rc = check_tokens(s, tokens);
  if (rc || tokens == 0) return rc;
  rc = check_ints({slots});
  if (!rc) rc = check_cache(k_pages, v_pages);
  if (!rc) rc = check_rows(s, k_out, "k_out");
  if (!rc) rc = check_rows(s, v_out, "v_out");
  if (!rc) rc = check_apart(s, tokens, s->kv_heads, k_out, "k_out");
  if (!rc) rc = check_apart(s, tokens, s->kv_heads, v_out, "v_out");
  if (rc) return rc;
  for (const Span& out : {span_of("k_out", s, k_out, tokens, s->kv_heads, WRITTEN), span_of("v_out", s, v_out, tokens, s->kv_heads, WRITTEN)}) {
    rc = check_disjoint({out, span_of("k_pages", k_pages, pages_bytes(s), READ), span_of("v_pages", v_pages, pages_bytes(s), READ),
                         span_of("slots", slots, size_t(tokens) * 4, READ)});
    if (rc) return rc;
  }
  if (rows_meet(s, k_out, v_out, tokens, s->kv_heads)) return fail(HEATKV_EINVAL, "k_out overlaps v_out");
  heatkv::PagedReadArgs a{};
  a.dtype = s->dtype;
  a.d = s->d;
  a.H = s->kv_heads;
  a.page_log2 = log2_of(s->page_size);
  a.num_pages = s->num_pages;
  a.kv_format = s->kv_format;
  a.tokens = tokens;
  a.slots = slots;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.k_out = k_out.data;
  a.v_out = v_out.data;
  a.k_token_stride = k_out.token_stride;
  a.k_head_stride = k_out.head_stride;
  a.v_token_stride = v_out.token_stride;
  a.v_head_stride = v_out.head_stride;
  return launched(heatkv::launch_paged_read(a, static_cast<hipStream_t>(stream)), "paged_read");
}

size_t heatkv_paged_tables_workspace_bytes(const heatkv_paged_shape* s) { return check_shape(s) ? 0 : tables_workspace_of(s).total; }

int heatkv_paged_fork(const heatkv_paged_shape* s, const int32_t* parent, const int32_t* lens, int32_t* lens_out, int32_t* holders,
                      int32_t* free_ring, const int32_t* free_span, int32_t* free_span_out, int32_t* table, int32_t* status,
                      void* ws, size_t ws_bytes, void* stream) {
  Tables t{s, lens, lens_out, holders, free_ring, free_span, free_span_out, table, status, ws, ws_bytes};
  int rc = t.check();
  if (!rc) rc = check_ints({parent});
  if (!rc) rc = t.check_apart_from({}, {span_of("parent", parent, size_t(s->batch) * 4, READ)});
  if (rc) return rc;
  heatkv::ForkArgs f{};
  f.t = t.args();
  f.parent = parent;
  return launched(heatkv::launch_paged_fork(f, static_cast<hipStream_t>(stream)), "paged_fork");
}

int heatkv_paged_assign_shared(const heatkv_paged_shape* s, const int32_t* keep, const int32_t* new_tokens, const int32_t* lens,
                               int32_t* lens_out, int32_t* holders, int32_t* free_ring, const int32_t* free_span,
                               int32_t* free_span_out, int32_t* table, int32_t* q_start, int32_t* slots, int64_t max_tokens,
                               int32_t* copy_from, int32_t* copy_to, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  Tables t{s, lens, lens_out, holders, free_ring, free_span, free_span_out, table, status, ws, ws_bytes};
  int rc = t.check();
  if (!rc) rc = check_tokens(max_tokens);
  if (!rc) rc = check_ints({keep, new_tokens, q_start, copy_from, copy_to});
  if (!rc && max_tokens > 0) rc = check_ints({slots});
  if (rc) return rc;
  const size_t row = size_t(s->batch) * 4, copies = row * s->page_size;
  rc = t.check_apart_from({span_of("q_start", q_start, row + 4, WRITTEN), span_of("slots", slots, size_t(max_tokens) * 4, WRITTEN),
                           span_of("copy_from", copy_from, copies, WRITTEN), span_of("copy_to", copy_to, copies, WRITTEN)},
                          {span_of("keep", keep, row, READ), span_of("new_tokens", new_tokens, row, READ)});
  if (rc) return rc;
  heatkv::AssignSharedArgs a{};
  a.t = t.args();
  a.keep = keep;
  a.new_tokens = new_tokens;
  a.q_start = q_start;
  a.slots = slots;
  a.copy_from = copy_from;
  a.copy_to = copy_to;
  a.max_tokens = max_tokens;
  a.take0 = t.at<int32_t>(t.w.per_row[0]);
  a.touch0 = t.at<int32_t>(t.w.per_row[1]);
  a.first = t.at<int32_t>(t.w.per_row[2]);
  a.copied = t.at<int32_t>(t.w.per_row[3]);
  return launched(heatkv::launch_paged_assign_shared(a, static_cast<hipStream_t>(stream)), "paged_assign_shared");
}

int heatkv_paged_compact(const heatkv_paged_shape* s, const uint8_t* kept, const int32_t* lens, int32_t* lens_out, int32_t* holders,
                         int32_t* free_ring, const int32_t* free_span, int32_t* free_span_out, int32_t* table, int32_t* move_from,
                         int32_t* move_to, int64_t max_moves, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  Tables t{s, lens, lens_out, holders, free_ring, free_span, free_span_out, table, status, ws, ws_bytes};
  int rc = t.check();
  if (!rc) rc = check_tokens(max_moves);
  if (!rc && max_moves > 0) rc = check_ints({move_from, move_to});
  if (rc) return rc;
  if (!kept || !aligned(kept, 16)) return fail(HEATKV_EINVAL, "kept must be 16-byte aligned and not null");
  const size_t list = size_t(max_moves) * 4;
  rc = t.check_apart_from({span_of("move_from", move_from, list, WRITTEN), span_of("move_to", move_to, list, WRITTEN)},
                          {span_of("kept", kept, size_t(s->batch) * s->max_pages * s->page_size, READ)});
  if (rc) return rc;
  heatkv::CompactArgs a{};
  a.t = t.args();
  a.kept = kept;
  a.move_from = move_from;
  a.move_to = move_to;
  a.max_moves = max_moves;
  a.tile = t.w.tile;
  a.tiles = t.w.tiles;
  a.take0 = t.at<int32_t>(t.w.per_row[0]);
  a.move0 = t.at<int32_t>(t.w.per_row[1]);
  a.first = t.at<int32_t>(t.w.per_row[2]);
  a.counts = t.at<int32_t>(t.w.counts);
  a.drops = t.at<int32_t>(t.w.drops);
  return launched(heatkv::launch_paged_compact(a, static_cast<hipStream_t>(stream)), "paged_compact");
}

}  // extern "C"
