// Paged cache: pages that several rows of the block table hold, and rows that lose tokens out of their middle.
//
//   fork     row b continues row parent[b]: its entries and length become those of that row
//   assign   a step of the allocator (paged_tables.hip) that leaves a page alone which another row holds too
//   compact  a row keeps the marked ones of its tokens, in order; the move of their rows is listed
//
// holders[page]: rows of the table that hold it.  A row that gains a page counts one up, one that loses it one down; the page
// whose count comes down to 0 is marked in a bitmap, and the last launch of a call puts the marked pages behind the ring's tail
// in ascending order.  Counts are whole numbers and marks are bits, so the result does not depend on the order in which
// workgroups come by.  What is gained is counted before what is lost, in a launch of its own: no count passes through 0 on
// the way.
//
// Each call is a few phases that are launches of their own; `Group` says which of how many workgroups one is.
//
// Bound: latency, of the launches and of a few round trips to memory in each.  A step of 64 beams (fork, assign, the rows of one layer, with
// the copy of the tables that it starts from) takes 26 us, of 512 samples 40; one request of 3000 tokens thinned out 16 us, 32 of 8192
// tokens 119 us, 94 of them the rows of one layer.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "paged.h"

namespace heatkv {

namespace {

constexpr int LANES = 1024, WAVES = LANES / 64;
constexpr int PER_LANE = paged::MAX_BATCH / LANES;
constexpr int FORK_LANES = 256, FORK_ENTRIES = paged::MAX_BATCH;  // lanes of a workgroup, entries of the table that it may have
// Entries that it has if the batch is not larger: few, as a workgroup goes through them alone.  512 samples 39.8 us, with 1024 42.3, with
// 4096 62.7.  Fork alone, with 512, 2048, 4096 (and the copy of the tables, 3.5): 512 rows of 128 columns 18, 30, 45 us, of 512 columns 22,
// 32, 47, of 2048 48, 43, 54; 1024 rows of 128 24, 32, 48, of 2048 81, 76, 74.  More than 2048 rows have one column with all of them: 4096
// rows of 128 columns 59, of 512 92, of 2048 277.
constexpr int FORK_TARGET = 512;
constexpr int EMIT_LANES = 256, CHUNK = 4096;         // tokens that a workgroup of compact looks at together

struct Group {
  int index, count;
};
__device__ __forceinline__ Group group() { return {static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x)}; }

// Words of TableArgs::state.  MISFIT: not 0 once a page was let go that nobody held, by its count.
enum State { HEAD, COUNT, TAKEN, STATUS, MOVES, MISFIT };

// Sum over the lanes up to this one: within rows of 16 lanes, then from row to row.
__device__ __forceinline__ int inclusive_scan(int v) {
#define HEATKV_STEP(control, rows) v += __builtin_amdgcn_update_dpp(0, v, control, rows, 0xf, false)
  HEATKV_STEP(0x111, 0xf);  // one lane up, then 2, 4 and 8
  HEATKV_STEP(0x112, 0xf);
  HEATKV_STEP(0x114, 0xf);
  HEATKV_STEP(0x118, 0xf);
  HEATKV_STEP(0x142, 0xa);  // lane 15 of a row to the next row: rows 1 and 3
  HEATKV_STEP(0x143, 0xc);  // lane 31 to rows 2 and 3
#undef HEATKV_STEP
  return v;
}

// Largest b in [0, n) with first[b] <= x; first[0] = 0, ascending.
__device__ __forceinline__ int find(const int* first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    (first[mid] <= x ? lo : hi) = mid;
  }
  return lo;
}

__device__ __forceinline__ bool ring_fits(const TableArgs& p, int head, int count) {
  return head >= 0 && head < p.num_pages && count >= 0 && count <= p.num_pages;
}
// Entry i behind the ring's head; i below num_pages.
__device__ __forceinline__ int ring_at(const TableArgs& p, int head, int i) {
  const unsigned at = static_cast<unsigned>(head) + static_cast<unsigned>(i);
  return p.ring[at < static_cast<unsigned>(p.num_pages) ? at : at - p.num_pages];
}
__device__ __forceinline__ int in_range(const TableArgs& p, int page) {
  return static_cast<int>(min(static_cast<unsigned>(page), static_cast<unsigned>(p.num_pages - 1)));
}
__device__ __forceinline__ int pages_of(const TableArgs& p, int tokens) {
  return static_cast<int>((static_cast<long long>(tokens) + (1 << p.page_log2) - 1) >> p.page_log2);
}
__device__ __forceinline__ long long most_tokens(const TableArgs& p) { return static_cast<long long>(p.max_pages) << p.page_log2; }

// A row no longer holds `page`.
__device__ __forceinline__ void let_go(const TableArgs& p, int page) {
  page = in_range(p, page);
  const int held = atomicSub(&p.holders[page], 1);
  if (held == 1) atomicOr(&p.gone[page >> 5], 1u << (page & 31));
  if (held < 1) p.state[MISFIT] = 1;  // whoever finds it
}
// A row holds `page`, fresh from the ring.
__device__ __forceinline__ void take(const TableArgs& p, int page) { p.holders[in_range(p, page)] = 1; }

__device__ __forceinline__ int gone_words(const TableArgs& p) { return (p.num_pages + 31) / 32; }
__device__ __forceinline__ void clear_gone(const TableArgs& p, Group g, int lanes) {
  for (int i = g.index * lanes + threadIdx.x; i < gone_words(p); i += g.count * lanes) p.gone[i] = 0;
}

// ---- the last phase of every call: marked pages into the ring, lengths and the ring's span ------------------------------

// Workgroup g of the grid takes `each_group` words of the bitmap, and counts those before for itself.  Its words are dealt to its
// wavefronts in equal stretches: marked pages are often next to one another.  66000 pages given back: 17 us by one workgroup, 5.2 by six.
constexpr int GIVE_WORDS = 512, GIVE_GROUPS = 64;  // words of a workgroup at least, workgroups at most

__device__ __forceinline__ void give_back(const TableArgs& p, Group g) {
  __shared__ int part[2][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int all_words = gone_words(p), each_group = (all_words + g.count - 1) / g.count;
  const int first = min(g.index * each_group, all_words), words = min(all_words - first, each_group), R = p.num_pages;
  const int head = p.state[HEAD], count = p.state[COUNT], taken = p.state[TAKEN], misfit = p.state[MISFIT];
  int before = 0;
  for (int i = tid; i < first; i += LANES) before += __popc(p.gone[i]);
  const int each = (words + WAVES - 1) / WAVES, w0 = min(wave * each, words), w1 = min(w0 + each, words);
  int mine = 0;
  for (int i = w0 + lane; i < w1; i += 64) mine += __popc(p.gone[first + i]);
  const int inc = inclusive_scan(mine), earlier = inclusive_scan(before);
  if (lane == 63) {
    part[0][wave] = inc;
    part[1][wave] = earlier;
  }
  __syncthreads();
  int at = 0, all = 0, all_before = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    all_before += part[1][i];
    at += i < wave ? part[0][i] : 0;
    all += part[0][i];
  }
  at += all_before;
  const int room = R - (count - taken);  // holders that fit the table and the ring never have more to give
  for (int k = w0; k < w1; k += 64) {
    const unsigned w = k + lane < w1 ? p.gone[first + k + lane] : 0;
    unsigned long long todo = __ballot(w != 0);
    while (todo) {  // two words, 64 pages, at a time
      const int from = __builtin_ctzll(todo) & ~1;
      todo &= ~(3ull << from);
      const unsigned long long bits = static_cast<unsigned>(__builtin_amdgcn_readlane(w, from)) |
                                      static_cast<unsigned long long>(static_cast<unsigned>(__builtin_amdgcn_readlane(w, from + 1))) << 32;
      const int i = at + __popcll(bits & ((1ull << lane) - 1));
      if ((bits >> lane & 1) && i < room) {
        unsigned to = static_cast<unsigned>(head) + static_cast<unsigned>(count) + static_cast<unsigned>(i);  // below 3 R < 2^32
        to -= to >= static_cast<unsigned>(R) ? R : 0;
        to -= to >= static_cast<unsigned>(R) ? R : 0;
        p.ring[to] = 32 * (first + k + from) + lane;
      }
      at += __popcll(bits);
    }
  }
  if (g.index == 0)
    for (int b = tid; b < p.batch; b += LANES) p.lens_out[b] = p.next[b];
  if (g.index == g.count - 1 && tid == 0) {
    const bool made = p.state[STATUS] == HEATKV_PAGED_OK;  // else the span may be anything, and stays
    const int next = head + taken;
    p.span_out[0] = !made || next < R ? next : next - R;
    p.span_out[1] = made ? count - taken + min(all_before + all, room) : count;
    if (made && (misfit || all_before + all > room)) p.status[0] = HEATKV_PAGED_BAD_HOLDERS;
  }
}

// Small calls are one workgroup and one launch, which has the workspace in LDS.
constexpr int SMALL_BATCH = 1024, SMALL_PAGES = 131072;
template <int BATCH, int PAGES>
struct Small {
  int state[8], next[BATCH];
  uint32_t gone[PAGES / 32];
  __device__ __forceinline__ void lend(TableArgs& p) {
    p.state = state;
    p.next = next;
    p.gone = gone;
  }
};

// ---- fork ---------------------------------------------------------------------------------------------------------------

// Parents, pages held and pages to be, of all rows, into LDS; every workgroup looks at all of them for itself.
struct ForkRows {
  short parent[paged::MAX_BATCH];
  int held[paged::MAX_BATCH];
};
__device__ __forceinline__ int fork_load(const ForkArgs& f, ForkRows& r) {
  const TableArgs& p = f.t;
  const int tid = threadIdx.x, B = p.batch;
  const long long most = most_tokens(p);
  bool bad_parent = false, bad_length = false;
  for (int b = tid; b < B; b += FORK_LANES) {
    const int parent = f.parent[b], len = p.lens[b];
    bad_parent = bad_parent || parent < -1 || parent >= B;
    bad_length = bad_length || len < 0 || len > most;
    r.parent[b] = static_cast<short>(parent);
    r.held[b] = pages_of(p, len);
  }
  const bool any_length = __syncthreads_or(bad_length), any_parent = __syncthreads_or(bad_parent);
  return any_length ? HEATKV_PAGED_BAD_LENGTH : any_parent ? HEATKV_PAGED_BAD_PARENT : HEATKV_PAGED_OK;
}
// A row's entry in a column before and after; -1: none.  Where they are equal nothing changes: most of what beams have in common.
struct Change {
  int before, after;
};
__device__ __forceinline__ Change fork_change(const TableArgs& p, const ForkRows& r, int b, int c) {
  const int parent = r.parent[b];
  Change x{-1, -1};
  if (parent == b) return x;
  if (c < r.held[b]) x.before = in_range(p, p.table[static_cast<long long>(b) * p.max_pages + c]);
  if (parent >= 0 && c < r.held[parent]) x.after = in_range(p, p.table[static_cast<long long>(parent) * p.max_pages + c]);
  if (x.before == x.after) x.before = x.after = -1;
  return x;
}

// Counts what rows gain.
__device__ __forceinline__ void fork_gains(const ForkArgs& f, Group g, int columns_log2) {
  const TableArgs& p = f.t;
  __shared__ ForkRows r;
  const int tid = threadIdx.x, B = p.batch;
  clear_gone(p, g, FORK_LANES);
  const int head = p.span[0], count = p.span[1];
  int status = fork_load(f, r);
  if (status == HEATKV_PAGED_OK && !ring_fits(p, head, count)) status = HEATKV_PAGED_BAD_FREE_LIST;
  if (g.index == 0) {
    for (int b = tid; b < B; b += FORK_LANES) p.next[b] = status ? p.lens[b] : r.parent[b] < 0 ? 0 : p.lens[r.parent[b]];
    if (tid == 0) {
      p.state[HEAD] = head;
      p.state[COUNT] = count;
      p.state[TAKEN] = 0;
      p.state[STATUS] = status;
      p.state[MISFIT] = 0;
      p.status[0] = status;
    }
  }
  if (status) return;
  for (int i = tid; i < B << columns_log2; i += FORK_LANES) {
    const Change x = fork_change(p, r, i >> columns_log2, (g.index << columns_log2) + (i & ((1 << columns_log2) - 1)));
    if (x.after >= 0) atomicAdd(&p.holders[x.after], 1);
  }
}

// A workgroup has some columns of all rows: it reads them before it writes any, and nobody else does either.
__device__ __forceinline__ void fork_rows(const ForkArgs& f, Group g, int columns_log2) {
  const TableArgs& p = f.t;
  __shared__ ForkRows r;
  __shared__ int after[FORK_ENTRIES];
  const int status = p.state[STATUS];
  fork_load(f, r);
  if (status) return;
  const int tid = threadIdx.x, c0 = g.index << columns_log2, entries = p.batch << columns_log2;
  for (int i = tid; i < entries; i += FORK_LANES) {
    const Change x = fork_change(p, r, i >> columns_log2, c0 + (i & ((1 << columns_log2) - 1)));
    after[i] = x.after;
    if (x.before >= 0) let_go(p, x.before);
  }
  __syncthreads();
  for (int i = tid; i < entries; i += FORK_LANES)
    if (after[i] >= 0) p.table[static_cast<long long>(i >> columns_log2) * p.max_pages + c0 + (i & ((1 << columns_log2) - 1))] = after[i];
}

__global__ __launch_bounds__(FORK_LANES) void paged_fork_gains_kernel(ForkArgs f, int columns_log2) { fork_gains(f, group(), columns_log2); }
__global__ __launch_bounds__(FORK_LANES) void paged_fork_rows_kernel(ForkArgs f, int columns_log2) { fork_rows(f, group(), columns_log2); }
// All phases by one workgroup.  A row's columns are dealt to 2^side_log2 lanes, up to a wavefront of them, `pieces` to each; a lane
// has up to SMALL_EACH entries of the table.  Few instructions for each are what counts: one compute unit has them all.  Beams in
// groups of four, with the copy of the tables that the measurement starts from (3.7 us), by one workgroup and by launches of many: 64 x
// 16 entries 7.7 and 16.3 us, 64 x 64 11.0 and 16.5, 64 x 128 14.8 and 18.4, 64 x 256 21.6 and 19.6, 1024 x 16 25.3 and 21.1.
constexpr int SMALL_EACH = 12;
__global__ __launch_bounds__(LANES) void paged_fork_small_kernel(ForkArgs f, int side_log2, int pieces) {
  __shared__ Small<SMALL_BATCH, SMALL_PAGES> s;
  __shared__ int lens[SMALL_BATCH];
  struct Row {
    int parent, held, gets;  // a row that stays as it is holds and gets nothing
  };
  __shared__ Row rows[SMALL_BATCH];
  s.lend(f.t);
  const TableArgs& p = f.t;
  const int tid = threadIdx.x, B = p.batch;
  const int head = p.span[0], count = p.span[1];
  clear_gone(p, {0, 1}, LANES);
  bool bad_parent = false, bad_length = false;
  int parent = -1, len = 0;
  if (tid < B) {
    parent = f.parent[tid];
    len = p.lens[tid];
    bad_parent = parent < -1 || parent >= B;
    bad_length = len < 0 || len > most_tokens(p);
    lens[tid] = len;
  }
  const bool any_length = __syncthreads_or(bad_length), any_parent = __syncthreads_or(bad_parent);
  const int status = any_length                   ? HEATKV_PAGED_BAD_LENGTH
                     : any_parent                 ? HEATKV_PAGED_BAD_PARENT
                     : !ring_fits(p, head, count) ? HEATKV_PAGED_BAD_FREE_LIST
                                                  : HEATKV_PAGED_OK;
  if (tid < B) {
    const int next = status ? len : parent < 0 ? 0 : lens[parent];
    const bool changes = !status && parent != tid;
    p.next[tid] = next;
    rows[tid] = {max(parent, 0), changes ? pages_of(p, len) : 0, changes ? pages_of(p, next) : 0};
  }
  if (tid == 0) {
    p.state[HEAD] = head;
    p.state[COUNT] = count;
    p.state[TAKEN] = 0;
    p.state[STATUS] = status;
    p.state[MISFIT] = 0;
    p.status[0] = status;
  }
  __syncthreads();
  if (!status) {
    const int step = LANES >> side_log2, first_row = tid >> side_log2, first_column = tid & ((1 << side_log2) - 1);
    int before[SMALL_EACH], after[SMALL_EACH];
    // Entry k of this lane, in rows row0, row0 + step, ..: visit(k, row, column, whether it exists)
    auto entries = [&](auto&& visit) {
      int row0 = 0, piece = 0;
#pragma unroll
      for (int k = 0; k < SMALL_EACH; ++k) {
        if (row0 >= B) break;
        visit(k, row0 + first_row, (piece << side_log2) + first_column);
        if (++piece == pieces) {
          piece = 0;
          row0 += step;
        }
      }
    };
#pragma unroll
    for (int k = 0; k < SMALL_EACH; ++k) before[k] = after[k] = -1;
    entries([&](int k, int b, int c) {
      if (b >= B) return;
      const Row r = rows[b];
      if (c < r.held) before[k] = p.table[b * p.max_pages + c];
      if (c < r.gets) after[k] = p.table[r.parent * p.max_pages + c];
    });
    entries([&](int k, int b, int c) {
      if (b >= B) return;
      const Row r = rows[b];
      before[k] = c < r.held ? in_range(p, before[k]) : -1;
      after[k] = c < r.gets ? in_range(p, after[k]) : -1;
      if (before[k] == after[k]) before[k] = after[k] = -1;
      if (after[k] >= 0) atomicAdd(&p.holders[after[k]], 1);
    });
    wait_vmcnt<0>();  // counted, before anything is counted down; and all entries have been read
    __syncthreads();
    int held_by[SMALL_EACH];
    entries([&](int k, int b, int c) {
      if (before[k] >= 0) held_by[k] = atomicSub(&p.holders[before[k]], 1);
      if (after[k] >= 0) p.table[b * p.max_pages + c] = after[k];
    });
    int least = 1;
#pragma unroll
    for (int k = 0; k < SMALL_EACH; ++k)
      if (before[k] >= 0) {
        if (held_by[k] == 1) atomicOr(&p.gone[before[k] >> 5], 1u << (before[k] & 31));
        least = min(least, held_by[k]);
      }
    if (least < 1) p.state[MISFIT] = 1;
  }
  __syncthreads();
  give_back(p, {0, 1});
}

__global__ __launch_bounds__(LANES) void paged_give_back_kernel(TableArgs p) { give_back(p, group()); }

// ---- assign -------------------------------------------------------------------------------------------------------------

// Sums over the requests before of N numbers that each lane has for its PER_LANE consecutive requests; `all`: of all.  Those of a
// wavefront's lanes are below 2^31 together.
template <int N>
__device__ __forceinline__ void scan_requests(const int (&sum)[N], long long (&before)[N], long long (&all)[N]) {
  __shared__ int part[N][WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int inc = inclusive_scan(sum[k]);
    before[k] = inc - sum[k];
    all[k] = 0;
    if (lane == 63) part[k][wave] = inc;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int x = part[k][w];
      if (w < wave) before[k] += x;
      all[k] += x;
    }
}

// What each request takes and lets go.  Columns from first[b] = ceil(keep / page) on, or from the one before where the new
// tokens would go onto a page that another row holds (copied[b]: that page, or -1): fresh pages up to ceil((keep + new) / page),
// what the row held there is let go.
__device__ __forceinline__ void assign_plan(const AssignSharedArgs& a, Group g) {
  const TableArgs& p = a.t;
  if (g.count > 1 && g.index > 0) return clear_gone(p, {g.index - 1, g.count - 1}, LANES);
  if (g.count == 1) clear_gone(p, g, LANES);
  const int tid = threadIdx.x, B = p.batch, page = 1 << p.page_log2;
  const int head = p.span[0], count = p.span[1];
  const long long most = most_tokens(p);
  const int per = (B + LANES - 1) / LANES;
  int first[PER_LANE], fresh[PER_LANE], touched[PER_LANE], come[PER_LANE], next[PER_LANE], old[PER_LANE];
  int sum[3] = {0, 0, 0};  // pages to take, columns to look at, tokens
  long long before[3], all[3];
  bool bad = false, many = false;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    first[i] = fresh[i] = touched[i] = come[i] = next[i] = 0;
    old[i] = -1;
    if (i >= per || b >= B) continue;
    const int len = p.lens[b], keep = a.keep[b], n = a.new_tokens[b];
    next[i] = len;
    if (len < 0 || len > most || keep < 0 || keep > len || n < 0 || static_cast<long long>(keep) + n > most) {
      bad = true;
      continue;
    }
    first[i] = pages_of(p, keep);
    many = many || n > a.max_tokens;
    come[i] = static_cast<int>(min(static_cast<long long>(n), a.max_tokens + 1));  // 2^22 + 1 at the most: 256 of them fit an int
    next[i] = keep + n;
    if (n > 0 && (keep & (page - 1))) {
      const int last = in_range(p, p.table[static_cast<long long>(b) * p.max_pages + first[i] - 1]);
      if (p.holders[last] > 1) {
        old[i] = last;
        --first[i];
      }
    }
    const int end = pages_of(p, keep + n);
    fresh[i] = end - first[i];
    touched[i] = max(end, pages_of(p, len)) - first[i];
  }
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    sum[0] += fresh[i];
    sum[1] += touched[i];
    sum[2] += come[i];
  }
  scan_requests(sum, before, all);
  const bool any_bad = __syncthreads_or(bad), any_many = __syncthreads_or(many);
  const int status = any_bad                      ? HEATKV_PAGED_BAD_LENGTH
                     : !ring_fits(p, head, count) ? HEATKV_PAGED_BAD_FREE_LIST
                     : any_many || all[2] > a.max_tokens ? HEATKV_PAGED_TOO_MANY_TOKENS
                     : all[0] > count             ? HEATKV_PAGED_NO_PAGES
                                                  : HEATKV_PAGED_OK;
  const bool ok = status == HEATKV_PAGED_OK;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    if (i >= per || b >= B) continue;
    a.take0[b] = ok ? static_cast<int>(before[0]) : 0;
    a.touch0[b] = ok ? static_cast<int>(before[1]) : 0;
    a.q_start[b] = ok ? static_cast<int>(before[2]) : 0;
    a.first[b] = first[i];
    a.copied[b] = ok ? old[i] : -1;
    p.next[b] = ok ? next[i] : p.lens[b];
    before[0] += fresh[i];
    before[1] += touched[i];
    before[2] += come[i];
  }
  if (tid == 0) {
    a.touch0[B] = ok ? static_cast<int>(all[1]) : 0;  // below 2^31: see check_tables()
    a.q_start[B] = ok ? static_cast<int>(all[2]) : 0;
    p.state[HEAD] = head;
    p.state[COUNT] = count;
    p.state[TAKEN] = ok ? static_cast<int>(all[0]) : 0;
    p.state[STATUS] = status;
    p.state[MISFIT] = 0;
    p.status[0] = status;
  }
}

// touch0, q0: those of `a`, in LDS.
__device__ __forceinline__ void assign_move(const AssignSharedArgs& a, Group g, const int* touch0, const int* q0) {
  const TableArgs& p = a.t;
  const int tid = threadIdx.x, B = p.batch, lp = p.page_log2, page = 1 << lp;
  const int touched = a.touch0[B], tokens = a.q_start[B], head = p.state[HEAD];
  const int at = g.index * LANES + tid, stride = g.count * LANES;
  auto row = [&](int b) { return p.table + static_cast<long long>(b) * p.max_pages; };
  for (int i = at; i < touched; i += stride) {
    const int b = find(touch0, B, i), nth = i - touch0[b], c = a.first[b] + nth;
    int* const entry = row(b) + c;
    if (c < pages_of(p, p.lens[b])) let_go(p, *entry);
    if (c < pages_of(p, p.next[b])) {
      const int fresh = ring_at(p, head, a.take0[b] + nth);
      *entry = fresh;
      take(p, fresh);
    }
  }
  for (long long t = at; t < a.max_tokens; t += stride) {
    int slot = -1;
    if (t < tokens) {
      const int b = find(q0, B, static_cast<int>(t));
      const int x = a.keep[b] + static_cast<int>(t) - q0[b], c = x >> lp, first = a.first[b];
      // a fresh entry of the table may be another workgroup's to write; those before the first are not written
      slot = ((c >= first ? ring_at(p, head, a.take0[b] + c - first) : row(b)[c]) << lp) + (x & (page - 1));
    }
    a.slots[t] = slot;
  }
  for (int i = at; i < B << lp; i += stride) {
    const int b = i >> lp, r = i & (page - 1), old = a.copied[b];
    const bool copy = old >= 0 && r < (a.keep[b] & (page - 1));
    a.copy_from[i] = copy ? (old << lp) + r : -1;
    a.copy_to[i] = copy ? (ring_at(p, head, a.take0[b]) << lp) + r : -1;
  }
}

__global__ __launch_bounds__(LANES) void paged_assign_plan_kernel(AssignSharedArgs a) { assign_plan(a, group()); }
__global__ __launch_bounds__(LANES) void paged_assign_move_kernel(AssignSharedArgs a) {
  __shared__ int touch0[paged::MAX_BATCH], q0[paged::MAX_BATCH];
  for (int b = threadIdx.x; b < a.t.batch; b += LANES) {
    touch0[b] = a.touch0[b];
    q0[b] = a.q_start[b];
  }
  __syncthreads();
  assign_move(a, group(), touch0, q0);
}

// All phases by one workgroup, what passes between them in LDS.
__global__ __launch_bounds__(LANES) void paged_assign_small_kernel(AssignSharedArgs a) {
  __shared__ Small<SMALL_BATCH, SMALL_PAGES> s;
  __shared__ int take0[SMALL_BATCH], touch0[SMALL_BATCH + 1], first[SMALL_BATCH], copied[SMALL_BATCH], q0[SMALL_BATCH + 1];
  int* const q_start = a.q_start;
  s.lend(a.t);
  a.take0 = take0;
  a.touch0 = touch0;
  a.first = first;
  a.copied = copied;
  a.q_start = q0;
  assign_plan(a, {0, 1});
  __syncthreads();
  for (int b = threadIdx.x; b <= a.t.batch; b += LANES) q_start[b] = q0[b];
  assign_move(a, {0, 1}, touch0, q0);
  __syncthreads();
  give_back(a.t, {0, 1});
}

// ---- compact ------------------------------------------------------------------------------------------------------------

// The tokens of request b that workgroup g looks at: a.tile of them from `first` on, as far as the request has any.
struct Stretch {
  int b, tile, first, end;
};
__device__ __forceinline__ Stretch stretch_of(const CompactArgs& a, Group g) {
  const int b = g.index / a.tiles, tile = g.index - b * a.tiles;
  const long long first = static_cast<long long>(tile) * a.tile;
  const long long len = min(static_cast<long long>(max(a.t.lens[b], 0)), most_tokens(a.t));
  return {b, tile, static_cast<int>(min(first, len)), static_cast<int>(min(first + a.tile, len))};
}

// Of every stretch: how many tokens are kept, and the first one that is not.
__device__ __forceinline__ void compact_count(const CompactArgs& a, Group g) {
  const TableArgs& p = a.t;
  __shared__ int part[2][EMIT_LANES / 64];
  clear_gone(p, g, EMIT_LANES);
  const Stretch s = stretch_of(a, g);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned char* const kept = a.kept + s.b * most_tokens(p);  // rows and stretches begin at multiples of 16 bytes
  int n = 0, drop = INT_MAX;
  for (int x = s.first + 16 * tid; x < s.end; x += 16 * EMIT_LANES) {
    const uint4 raw = ldg16(kept + x);
    const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // 0x80 in each byte that is not 0
      unsigned any = ((w[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu | w[i]) & 0x80808080u;
      const int left = s.end - (x + 4 * i);
      const unsigned real = left >= 4 ? 0x80808080u : left > 0 ? 0x80808080u & ((1u << 8 * left) - 1) : 0;
      any &= real;
      n += __popc(any);
      const unsigned none = any ^ real;
      if (none) drop = min(drop, x + 4 * i + (__builtin_ctz(none) >> 3));
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    n += __shfl_xor(n, m, 64);
    drop = min(drop, __shfl_xor(drop, m, 64));
  }
  if (lane == 0) {
    part[0][wave] = n;
    part[1][wave] = drop;
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < EMIT_LANES / 64; ++i) {
      n += part[0][i];
      drop = min(drop, part[1][i]);
    }
    a.counts[g.index] = n;
    a.drops[g.index] = drop;
  }
}

// Requests with kept tokens behind a dropped one take fresh pages for all from the page of that one on.
__device__ __forceinline__ void compact_plan(const CompactArgs& a) {
  const TableArgs& p = a.t;
  __shared__ int totals[paged::MAX_BATCH], leads[paged::MAX_BATCH];
  const int tid = threadIdx.x, B = p.batch;
  const int head = p.span[0], count = p.span[1];
  const long long most = most_tokens(p);
  // `side` lanes to a request, which share its stretches
  int side = 1;
  while (side < 64 && side < a.tiles) side *= 2;
  for (int b = tid / side; b < (B + LANES / side - 1) / (LANES / side) * (LANES / side); b += LANES / side) {
    const int len = b < B ? p.lens[b] : 0;
    int n = 0, drop = INT_MAX;
    if (b < B && len > 0 && len <= most)
      for (int i = tid % side; static_cast<long long>(i) * a.tile < len; i += side) {
        n += a.counts[b * a.tiles + i];
        drop = min(drop, a.drops[b * a.tiles + i]);
      }
    for (int m = 1; m < side; m *= 2) {
      n += __shfl_xor(n, m, 64);
      drop = min(drop, __shfl_xor(drop, m, 64));
    }
    if (b < B && tid % side == 0) {
      totals[b] = n;
      leads[b] = min(drop, len);
    }
  }
  __syncthreads();
  const int per = (B + LANES - 1) / LANES;
  int first[PER_LANE], fresh[PER_LANE], moves[PER_LANE], total[PER_LANE];
  int sum[2] = {0, 0};  // pages to take, rows to move
  long long before[2], all[2];
  bool many = false;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    first[i] = fresh[i] = moves[i] = total[i] = 0;
    if (i >= per || b >= B) continue;
    const int len = p.lens[b];
    if (len < 0 || len > most) {
      bad = true;
      continue;
    }
    total[i] = totals[b];
    const bool cut = total[i] == leads[b];  // only the last tokens go, or none
    first[i] = cut ? pages_of(p, total[i]) : leads[b] >> p.page_log2;
    fresh[i] = pages_of(p, total[i]) - first[i];
    moves[i] = cut ? 0 : total[i] - (first[i] << p.page_log2);
    many = many || moves[i] > a.max_moves;
    sum[0] += fresh[i];
    sum[1] += static_cast<int>(min(static_cast<long long>(moves[i]), a.max_moves + 1));  // see assign_plan()
  }
  scan_requests(sum, before, all);
  const bool any_bad = __syncthreads_or(bad), any_many = __syncthreads_or(many);
  const int status = any_bad                      ? HEATKV_PAGED_BAD_LENGTH
                     : !ring_fits(p, head, count) ? HEATKV_PAGED_BAD_FREE_LIST
                     : any_many || all[1] > a.max_moves ? HEATKV_PAGED_TOO_MANY_TOKENS
                     : all[0] > count             ? HEATKV_PAGED_NO_PAGES
                                                  : HEATKV_PAGED_OK;
  const bool ok = status == HEATKV_PAGED_OK;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    const int b = tid * per + i;
    if (i >= per || b >= B) continue;
    a.take0[b] = ok ? static_cast<int>(before[0]) : 0;
    a.move0[b] = ok && moves[i] > 0 ? static_cast<int>(before[1]) : -1;
    a.first[b] = first[i];
    p.next[b] = ok ? total[i] : p.lens[b];
    before[0] += fresh[i];
    before[1] += moves[i];
  }
  if (tid == 0) {
    p.state[HEAD] = head;
    p.state[COUNT] = count;
    p.state[TAKEN] = ok ? static_cast<int>(all[0]) : 0;
    p.state[STATUS] = status;
    p.state[MISFIT] = 0;
    p.state[MOVES] = ok ? static_cast<int>(all[1]) : 0;
    p.status[0] = status;
  }
}

// Tables and the list of moves.  A workgroup reads the entries of its stretch's columns before it writes them, and nobody else
// reads or writes these.
__device__ __forceinline__ void compact_emit(const CompactArgs& a, Group g) {
  const TableArgs& p = a.t;
  constexpr int COLUMNS = CHUNK / paged::GRANULE, GROUP_WAVES = EMIT_LANES / 64, ROUNDS = CHUNK / EMIT_LANES;
  __shared__ int entries[COLUMNS], fresh[COLUMNS + 1];  // of the chunk's columns, of those that its tokens go to
  __shared__ int part[GROUP_WAVES], base_part[GROUP_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lp = p.page_log2, page = 1 << lp;
  const int total_moves = p.state[MOVES], status = p.state[STATUS], head = p.state[HEAD];
  auto no_moves = [&](int from) {  // behind the last move
    for (long long m = from + static_cast<long long>(g.index) * EMIT_LANES + tid; m < a.max_moves;
         m += static_cast<long long>(g.count) * EMIT_LANES)
      a.move_from[m] = a.move_to[m] = -1;
  };
  const Stretch s = stretch_of(a, g);
  const int first = a.first[s.b], take0 = a.take0[s.b], move0 = a.move0[s.b];
  const int held = pages_of(p, p.lens[s.b]), want = pages_of(p, p.next[s.b]);
  if (status || s.first >= s.end || (static_cast<long long>(first) << lp) >= s.end) {  // nothing, or all of it stays where it is
    no_moves(total_moves);
    return;
  }
  const unsigned char* const kept = a.kept + s.b * most_tokens(p);
  int* const row = p.table + static_cast<long long>(s.b) * p.max_pages;
  // tokens that are kept before the stretch
  int base = 0;
  for (int i = tid; i < s.tile; i += EMIT_LANES) base += a.counts[g.index - s.tile + i];
  base = inclusive_scan(base);
  if (lane == 63) base_part[wave] = base;
  for (int x0 = s.first; x0 < s.end; x0 += CHUNK) {
    // a wavefront has 64 tokens a round, next to one another
    const int w0 = x0 + wave * (CHUNK / GROUP_WAVES) + lane;
    unsigned char byte[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) byte[i] = w0 + 64 * i < s.end ? kept[w0 + 64 * i] : 0;
    const int c0 = x0 >> lp, columns = CHUNK >> lp, c = c0 + tid;
    const bool changes = tid < columns && c >= first && c < held;
    const int entry = changes ? in_range(p, row[c]) : 0;
    __syncthreads();  // base_part is there; the arrays are free again
    if (x0 == s.first) {
      base = 0;
#pragma unroll
      for (int i = 0; i < GROUP_WAVES; ++i) base += base_part[i];
    }
    const int to0 = max(base >> lp, first);  // column of the chunk's first token that moves
    for (int i = tid; i <= columns; i += EMIT_LANES)
      if (to0 + i < want) fresh[i] = in_range(p, ring_at(p, head, take0 + to0 + i - first));
    if (changes) {
      entries[tid] = entry;
      let_go(p, entry);
      if (c < want) {
        const int mine = ring_at(p, head, take0 + c - first);
        row[c] = mine;
        take(p, mine);
      }
    }
    unsigned long long mask[ROUNDS];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      mask[i] = __ballot(byte[i] != 0);
      mine += __popcll(mask[i]);
    }
    if (lane == 0) part[wave] = mine;
    __syncthreads();
    int to = base;
#pragma unroll
    for (int i = 0; i < GROUP_WAVES; ++i) {
      to += i < wave ? part[i] : 0;
      base += part[i];
    }
    if (move0 < 0) continue;  // only its last tokens go
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      const int x = w0 + 64 * i;
      if ((mask[i] >> lane & 1) && (x >> lp) >= first) {
        const int y = to + __popcll(mask[i] & ((1ull << lane) - 1)), m = move0 + y - (first << lp);
        a.move_from[m] = (entries[(x >> lp) - c0] << lp) + (x & (page - 1));
        a.move_to[m] = (fresh[(y >> lp) - to0] << lp) + (y & (page - 1));
      }
      to += __popcll(mask[i]);
    }
  }
  no_moves(total_moves);
}

__global__ __launch_bounds__(EMIT_LANES) void paged_compact_count_kernel(CompactArgs a) { compact_count(a, group()); }
__global__ __launch_bounds__(LANES) void paged_compact_plan_kernel(CompactArgs a) { compact_plan(a); }
__global__ __launch_bounds__(EMIT_LANES) void paged_compact_emit_kernel(CompactArgs a) { compact_emit(a, group()); }

// All phases by one workgroup: a lane has 16 tokens next to one another, on one page.  Every other token goes, as above: 4 requests of up
// to 4096 tokens 13.1 us and by launches of many 19.7, 256 of 64 tokens 13.3 and 19.1.
constexpr int SMALL_TOKENS = 16 * LANES, THIN_BATCH = 256, THIN_PAGES = 65536;
__global__ __launch_bounds__(LANES) void paged_compact_small_kernel(CompactArgs a) {
  __shared__ Small<THIN_BATCH, THIN_PAGES> s;
  __shared__ int kept_before[LANES], entries[LANES], part[WAVES];
  __shared__ int take0[THIN_BATCH], move0[THIN_BATCH], first[THIN_BATCH], leads[THIN_BATCH];
  __shared__ unsigned short stays[SMALL_TOKENS];  // tokens that move, by their places in `kept`
  s.lend(a.t);
  const TableArgs& p = a.t;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = p.batch, lp = p.page_log2, page = 1 << lp;
  const int head = p.span[0], count = p.span[1], width = p.max_pages << lp;
  clear_gone(p, {0, 1}, LANES);
  // this lane's tokens
  const bool real = 16 * tid < B * width;
  const int b = real ? 16 * tid / width : 0, x0 = 16 * tid - b * width;
  const int here = real ? min(max(max(p.lens[b], 0) - x0, 0), 16) : 0;
  unsigned mask = 0;
  if (here > 0) {
    const uint4 raw = ldg16(a.kept + 16 * tid);
    const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) mask |= (w[i >> 2] >> 8 * (i & 3) & 0xff) ? 1u << i : 0;
    mask &= (1u << here) - 1;
  }
  int entry = 0;
  if (here > 0) entry = in_range(p, p.table[b * p.max_pages + (x0 >> lp)]);
  if (tid < B) leads[tid] = INT_MAX;
  const int mine = __popc(mask), inc = inclusive_scan(mine);
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  int earlier = inc - mine, whole = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    earlier += w < wave ? part[w] : 0;
    whole += part[w];
  }
  kept_before[tid] = earlier;
  entries[tid] = entry;
  const unsigned none = ~mask & ((1u << here) - 1);
  if (none) atomicMin(&leads[b], x0 + __builtin_ctz(none));
  __syncthreads();
  // the requests, one to a lane
  int fresh = 0, moves = 0, total = 0, from = 0;
  bool bad = false;
  if (tid < B) {
    const int n = p.lens[tid], end = (tid + 1) * width / 16;
    bad = n < 0 || n > width;
    if (!bad) {
      total = (end < LANES ? kept_before[end] : whole) - kept_before[tid * width / 16];
      const int lead = min(leads[tid], n);
      const bool cut = total == lead;
      from = cut ? pages_of(p, total) : lead >> lp;
      fresh = pages_of(p, total) - from;
      moves = cut ? 0 : total - (from << lp);
    }
  }
  const int sum[2] = {fresh, moves};
  long long before[2], all[2];
  scan_requests(sum, before, all);
  const bool any_bad = __syncthreads_or(bad);
  const int status = any_bad                      ? HEATKV_PAGED_BAD_LENGTH
                     : !ring_fits(p, head, count) ? HEATKV_PAGED_BAD_FREE_LIST
                     : all[1] > a.max_moves       ? HEATKV_PAGED_TOO_MANY_TOKENS
                     : all[0] > count             ? HEATKV_PAGED_NO_PAGES
                                                  : HEATKV_PAGED_OK;
  if (tid < B) {
    take0[tid] = static_cast<int>(before[0]);
    move0[tid] = moves > 0 ? static_cast<int>(before[1]) : -1;
    first[tid] = from;
    p.next[tid] = status ? p.lens[tid] : total;
  }
  const int listed = status ? 0 : static_cast<int>(all[1]);
  if (tid == 0) {
    p.state[HEAD] = head;
    p.state[COUNT] = count;
    p.state[TAKEN] = status ? 0 : static_cast<int>(all[0]);
    p.state[STATUS] = status;
    p.state[MISFIT] = 0;
    p.status[0] = status;
  }
  __syncthreads();
  const int c = x0 >> lp, start = first[b];
  if (!status && here > 0 && c >= start) {
    if ((x0 & (page - 1)) == 0) {
      let_go(p, entry);
      if (c < pages_of(p, p.next[b])) {
        const int page_now = ring_at(p, head, take0[b] + c - start);
        p.table[b * p.max_pages + c] = page_now;
        take(p, page_now);
      }
    }
    if (move0[b] >= 0) {
      int m = move0[b] + earlier - kept_before[b * width / 16] - (start << lp);
      for (unsigned bits = mask; bits; bits &= bits - 1) stays[m++] = static_cast<unsigned short>(16 * tid + __builtin_ctz(bits));
    }
  }
  __syncthreads();
  for (int m = tid; m < listed; m += LANES) {
    const int at = stays[m], request = at / width, y = m - move0[request] + (first[request] << lp);
    a.move_from[m] = (entries[at >> 4] << lp) + (at & (page - 1));  // `width` is a multiple of the page
    a.move_to[m] = (in_range(p, ring_at(p, head, take0[request] + (y >> lp) - first[request])) << lp) + (y & (page - 1));
  }
  for (long long m = listed + tid; m < a.max_moves; m += LANES) a.move_from[m] = a.move_to[m] = -1;
  __syncthreads();
  give_back(p, {0, 1});
}

hipError_t launch_give_back(const TableArgs& p, hipStream_t stream) {
  const int groups = std::min(((p.num_pages + 31) / 32 + GIVE_WORDS - 1) / GIVE_WORDS, GIVE_GROUPS);
  hipLaunchKernelGGL(paged_give_back_kernel, dim3(groups), dim3(LANES), 0, stream, p);
  return hipGetLastError();
}

// Small enough for one workgroup that has the workspace in LDS.
template <int BATCH, int PAGES>
bool fits(const TableArgs& p) { return p.batch <= BATCH && p.num_pages <= PAGES; }

}  // namespace

hipError_t launch_paged_fork(const ForkArgs& f, hipStream_t stream) {
  int side_log2 = 0;
  while (side_log2 < 6 && 1 << side_log2 < f.t.max_pages) ++side_log2;
  const long long pieces = ((static_cast<long long>(f.t.max_pages) - 1) >> side_log2) + 1, step = LANES >> side_log2;
  if (fits<SMALL_BATCH, SMALL_PAGES>(f.t) && (f.t.batch + step - 1) / step * pieces <= SMALL_EACH) {
    hipLaunchKernelGGL(paged_fork_small_kernel, dim3(1), dim3(LANES), 0, stream, f, side_log2, static_cast<int>(pieces));
    return hipGetLastError();
  }
  int columns_log2 = 6;
  while (columns_log2 > 0 && f.t.batch << columns_log2 > FORK_TARGET) --columns_log2;
  const unsigned groups = static_cast<unsigned>((f.t.max_pages + (1 << columns_log2) - 1) >> columns_log2);
  hipLaunchKernelGGL(paged_fork_gains_kernel, dim3(groups), dim3(FORK_LANES), 0, stream, f, columns_log2);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(paged_fork_rows_kernel, dim3(groups), dim3(FORK_LANES), 0, stream, f, columns_log2);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_give_back(f.t, stream);
}

hipError_t launch_paged_assign_shared(const AssignSharedArgs& a, hipStream_t stream) {
  // A token each, most of them to pages that are shared, as above: 64 requests 9.4 us by one workgroup and 12.9 by launches of many, 512
  // requests 12.3 and 15.1.  The limits are of what it goes through alone: tokens, copies, entries of the table that may all be let go.
  const long long copies = static_cast<long long>(a.t.batch) << a.t.page_log2;
  if (fits<SMALL_BATCH, SMALL_PAGES>(a.t) && a.max_tokens <= 4 * LANES && copies <= 8 * LANES &&
      static_cast<long long>(a.t.batch) * a.t.max_pages <= 32 * LANES) {
    hipLaunchKernelGGL(paged_assign_small_kernel, dim3(1), dim3(LANES), 0, stream, a);
    return hipGetLastError();
  }
  const int words = (a.t.num_pages + 31) / 32;
  hipLaunchKernelGGL(paged_assign_plan_kernel, dim3(1 + std::min((words + LANES - 1) / LANES, 64)), dim3(LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  const long long work = std::max(a.max_tokens, copies);
  const auto groups = static_cast<unsigned>(std::min<long long>((work + LANES - 1) / LANES + a.t.batch / 32, 128));
  hipLaunchKernelGGL(paged_assign_move_kernel, dim3(groups), dim3(LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_give_back(a.t, stream);
}

hipError_t launch_paged_compact(const CompactArgs& a, hipStream_t stream) {
  if (fits<THIN_BATCH, THIN_PAGES>(a.t) && (static_cast<long long>(a.t.batch) * a.t.max_pages << a.t.page_log2) <= SMALL_TOKENS) {
    hipLaunchKernelGGL(paged_compact_small_kernel, dim3(1), dim3(LANES), 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(a.t.batch) * a.tiles);
  hipLaunchKernelGGL(paged_compact_count_kernel, grid, dim3(EMIT_LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(paged_compact_plan_kernel, dim3(1), dim3(LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(paged_compact_emit_kernel, grid, dim3(EMIT_LANES), 0, stream, a);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_give_back(a.t, stream);
}

}  // namespace heatkv
