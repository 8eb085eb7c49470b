// How a launch's work is dealt to workgroups when the lengths are on the device.
//
// A segment is a tile of query rows of a request and kv head, and has a weight, about proportional to the keys that it walks
// over.  A share is the weight of all segments over the workgroups that are resident at a time.  Two ways:
//
// Along a line, on which all segments lie (requests in order, of each the kv heads, of each the tiles): workgroup w takes the
// stretch [w share, (w + 1) share) of it.  Any mix of lengths is dealt evenly, with a grid that depends on nothing that the
// host does not know.  A segment that crosses from one share into another is computed in parts.
//
// By pieces: a segment is cut into as many equal parts as its request's mean weight is shares, and a workgroup takes one.
// They come as workgroups become free, the last tiles of a request first, which are the heaviest with a causal limit.  Parts
// are fewer than on the line, and no workgroup has two things to do one after the other.
//
// The steps of a part are in proportion to its weight; a second launch joins parts, in order.  Light segments are not cut.
// Every workgroup finds its part by a scan over the requests (a round of loads; for up to 64 requests within the wavefront).
#pragma once

#include "paged.h"

namespace heatkv {
namespace paged {

constexpr int STEP_WEIGHT = 32;  // of a step of KEYS keys; 2^25 steps at most: a weight is below 2^31

// What a request adds to the line, for each kv head: `tiles` segments of weights w0 + t dw.
struct Load {
  int tiles, w0, dw;  // tiles 0: none of this launch's requests
  __device__ __forceinline__ long long upto(int t) const {  // the first t segments
    return static_cast<long long>(t) * w0 + static_cast<long long>(t) * (t - 1) / 2 * dw;
  }
  __device__ __forceinline__ long long weight(int t) const { return w0 + static_cast<long long>(t) * dw; }
};
template <int ROWS, int KEYS>
__device__ __forceinline__ Load load_of(const AttendParams& p, int q0, int q1, int len) {
  const Cache& c = p.c;
  q0 = min(max(q0, 0), c.tokens);
  const int n_new = min(max(q1, q0), c.tokens) - q0, rows = n_new * c.G;
  Load l{0, STEP_WEIGHT, 0};
  if (rows <= p.least_rows || rows > p.most_rows) return l;
  l.tiles = (rows + ROWS - 1) / ROWS;
  len = min(max(len, 0), c.max_pages << c.page_log2);
  if (p.selected) {  // no more than a tile's tokens can have chosen between them
    const int tokens = min(min(ROWS, (ROWS - 1) / c.G + 2), n_new);
    len = min(len, tokens * p.top << c.page_log2);
  } else if (c.causal) {  // the last row of a tile sees ROWS / G keys more than that of the tile before
    l.dw = ROWS * STEP_WEIGHT / KEYS / c.G;
    len = max(len - n_new + min(n_new, ROWS / c.G), 0);
  }
  l.w0 = max((len + KEYS - 1) / KEYS, 1) * STEP_WEIGHT;
  return l;
}

// A number that all lanes have, in scalar registers.
__device__ __forceinline__ long long uniform(long long x) {
  const int lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return static_cast<long long>(hi) << 32 | static_cast<unsigned>(lo);
}

// n / d of numbers that are not negative: the 64-bit division takes several times the instructions of the 32-bit one.
__device__ __forceinline__ long long quotient(long long n, long long d) {
  if (((n | d) >> 31) == 0) return static_cast<unsigned>(n) / static_cast<unsigned>(d);
  return n / d;
}

struct Scratch {  // LDS
  long long sums[4], first;
  int b;
};

template <int ROWS, int KEYS>
__device__ __forceinline__ Load request_load(const AttendParams& p, int b) {
  return load_of<ROWS, KEYS>(p, uniform_load(p.c.q_start, b), uniform_load(p.c.q_start, b + 1), uniform_load(p.c.lens, b));
}

// The requests' loads, consecutive ones to each lane of the workgroup; up to 64 requests: one to each lane of every wavefront.
template <int ROWS, int KEYS>
struct Requests {
  const AttendParams& p;
  const bool narrow;
  const int first, count;  // this lane's
  Load own;                // of the first
  __device__ __forceinline__ Requests(const AttendParams& params)
      : p(params),
        narrow(params.c.batch <= 64),
        first(narrow ? threadIdx.x & 63 : static_cast<int>(threadIdx.x) * ((params.c.batch + 255) / 256)),
        count(narrow ? 1 : (params.c.batch + 255) / 256) {
    own = load(first);
  }
  __device__ __forceinline__ Load load(int b) const {
    if (b >= p.c.batch) return Load{0, STEP_WEIGHT, 0};
    return load_of<ROWS, KEYS>(p, p.c.q_start[b], p.c.q_start[b + 1], p.c.lens[b]);
  }
  template <class Cost>
  __device__ __forceinline__ long long mine(const Cost& cost) const {
    long long sum = cost(own);
    for (int i = 1; i < count; ++i) sum += cost(load(first + i));
    return sum;
  }
  // Sum of `v` over the lanes up to this one, and over all of them.  Between two calls with the same scratch: a barrier.
  __device__ __forceinline__ long long scan(long long v, Scratch& scratch, long long& all) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const long long u = __shfl_up(v, d, 64);
      if (lane >= d) v += u;
    }
    if (narrow) {
      all = last_lane(v);
      return v;
    }
    if (lane == 63) scratch.sums[wave] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long x = scratch.sums[i];
      if (i < wave) v += x;
      all += x;
    }
    __syncthreads();
    all = uniform(all);
    return v;
  }
  // The request that holds position `at`, and where it begins; upto, mine as above.
  template <class Cost>
  __device__ __forceinline__ int find(long long at, long long upto, long long mine, const Cost& cost, Scratch& scratch,
                                      long long& begins) const {
    if (narrow) {
      const int b = min(static_cast<int>(__popcll(__ballot(upto <= at))), 63);
      begins = lane_of(upto - mine, b);
      return b;
    }
    if (at < upto && at >= upto - mine) {  // one lane
      long long x = upto - mine;
      for (int i = 0; i < count; ++i) {
        const long long n = cost(load(first + i));
        if (at < x + n) {
          scratch.first = x;
          scratch.b = first + i;
          break;
        }
        x += n;
      }
    }
    __syncthreads();
    begins = uniform(scratch.first);
    return __builtin_amdgcn_readfirstlane(scratch.b);
  }
  // The load of request b, as every lane's own.
  __device__ __forceinline__ Load found(int b) const {
    if (!narrow) return request_load<ROWS, KEYS>(p, b);
    return Load{__builtin_amdgcn_readlane(own.tiles, b), __builtin_amdgcn_readlane(own.w0, b), __builtin_amdgcn_readlane(own.dw, b)};
  }
  static __device__ __forceinline__ long long lane_of(long long x, int l) {
    const int lo = __builtin_amdgcn_readlane(static_cast<int>(x), l), hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), l);
    return static_cast<long long>(hi) << 32 | static_cast<unsigned>(lo);
  }
  static __device__ __forceinline__ long long last_lane(long long x) { return lane_of(x, 63); }
};

// A part of a segment, in units of its weight; the whole segment: from == 0, to == weight.
struct Part {
  int b, h, t;
  long long from, to, weight;
};

// What the join has to know; written by every workgroup.  parts > 0: the border between its share and the one before cuts a
// segment (and no earlier border does); parts < 0: its piece is the first of -parts; 0: neither.
__device__ __forceinline__ void write_border(const AttendParams& p, int w, const Border& x) {
  if (p.parts.borders && threadIdx.x == 0) p.parts.borders[w] = x;
}

// The piece of workgroup w, by all of its 256 lanes; false: there is none.  Pieces of a segment lie H workgroups apart.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool find_piece(const AttendParams& p, const Requests<ROWS, KEYS>& requests, int w, long long share,
                                           Scratch& scratch, Part& part) {
  auto cuts = [&](const Load& l) { return l.tiles ? static_cast<int>(quotient(quotient(l.upto(l.tiles), l.tiles) + share - 1, share)) : 0; };
  auto cost = [&](const Load& l) { return static_cast<long long>(l.tiles) * cuts(l) * p.c.H; };
  const long long mine = requests.mine(cost);
  long long all, first;
  const long long upto = requests.scan(mine, scratch, all);
  if (w >= all) {
    write_border(p, w, Border{0, 0, 0, 0});
    return false;
  }
  part.b = requests.find(w, upto, mine, cost, scratch, first);
  const Load l = requests.found(part.b);
  const int n = cuts(l), rel = static_cast<int>(w - first), i = rel / p.c.H, tile = i / n;
  part.h = rel - i * p.c.H;
  part.t = l.tiles - 1 - tile;
  part.from = i - tile * n;
  part.to = part.from + 1;
  part.weight = n;
  // Parts behind the grid's end: of a q_start that is not ascending only.
  const bool joins = n > 1 && part.from == 0 && w + (n - 1ll) * p.c.H < p.parts.grid;
  write_border(p, w, Border{part.b, part.h, part.t, joins ? -n : 0});
  return true;
}
template <int ROWS, int KEYS>
__device__ __forceinline__ long long total_weight(const AttendParams& p, const Requests<ROWS, KEYS>& requests, Scratch& scratch,
                                                  long long& upto, long long& mine) {
  mine = requests.mine([&](const Load& l) { return l.upto(l.tiles) * p.c.H; });
  long long total;
  upto = requests.scan(mine, scratch, total);
  return total;
}
template <int ROWS, int KEYS>
__device__ __forceinline__ long long total_segments(const AttendParams& p, const Requests<ROWS, KEYS>& requests, Scratch& scratch) {
  long long count;
  requests.scan(requests.mine([&](const Load& l) { return static_cast<long long>(l.tiles) * p.c.H; }), scratch, count);
  return count;
}
__device__ __forceinline__ long long share_of(const AttendParams& p, long long total, long long shares) {
  return max(quotient(total + shares - 1, shares), static_cast<long long>(p.least_weight));
}

// By pieces only: whole segments from whole_from on, or where the workspace has no place for parts.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool only_piece(const AttendParams& p, int w, Scratch& scratch, Part& part) {
  const Requests<ROWS, KEYS> requests(p);
  long long upto, mine;
  const long long total = total_weight(p, requests, scratch, upto, mine);
  const bool whole = !p.parts.borders || total_segments(p, requests, scratch) >= p.whole_from;
  return find_piece(p, requests, w, whole ? total + 1 : share_of(p, total, p.workgroups), scratch, part);
}

struct Place {
  long long pos, stop;  // on the line; pos >= stop: nothing (more) to do
  int b, h, t;          // the segment at pos
  long long off;        // pos in it
  Load load;            // of request b
};
// The place of workgroup w on the line, by all lanes.
template <int ROWS, int KEYS>
__device__ __forceinline__ Place find_place(const AttendParams& p, const Requests<ROWS, KEYS>& requests, int w, long long total,
                                            long long upto, long long mine, Scratch& scratch) {
  const long long share = share_of(p, total, p.workgroups);
  Place at{};
  at.pos = w * share;
  at.stop = min(at.pos + share, total);
  Border border{0, 0, 0, 0};
  if (at.pos < total && w < p.workgroups) {
    long long first;
    at.b = requests.find(at.pos, upto, mine, [&](const Load& l) { return l.upto(l.tiles) * p.c.H; }, scratch, first);
    at.load = requests.found(at.b);
    const long long rel = at.pos - first, per_head = at.load.upto(at.load.tiles);
    at.h = static_cast<int>(quotient(rel, per_head));
    const long long in_head = rel - at.h * per_head;
    int below = 0, above = at.load.tiles;  // the last tile that begins at in_head or before
    while (above - below > 1) {
      const int mid = (below + above) >> 1;
      (at.load.upto(mid) <= in_head ? below : above) = mid;
    }
    at.t = below;
    at.off = in_head - at.load.upto(below);
    const long long weight = at.load.weight(at.t);
    border = Border{at.b, at.h, at.t, 0};
    if (at.off > 0 && at.off <= share && weight > p.cut_from)
      border.parts = 1 + static_cast<int>(quotient(weight - at.off + share - 1, share));
  } else {
    at.stop = at.pos;
  }
  write_border(p, w, border);
  return at;
}

// The part of the segment at pos that is this workgroup's; advances the place behind it.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool next_part(const AttendParams& p, Place& at, Part& part) {
  while (at.pos < at.stop) {
    const long long weight = at.load.weight(at.t);
    part = {at.b, at.h, at.t, at.off, min(weight, at.off + (at.stop - at.pos)), weight};
    if (weight <= p.cut_from) part.to = weight;
    at.pos += part.to - part.from;
    at.off = 0;
    if (part.to == weight && ++at.t == at.load.tiles) {
      at.t = 0;
      if (++at.h == p.c.H && at.pos < at.stop) {  // there is another request with a load
        at.h = 0;
        do {
          at.load = request_load<ROWS, KEYS>(p, ++at.b);
        } while (at.load.tiles == 0 && at.b + 1 < p.c.batch);
      }
    }
    if (weight > p.cut_from || part.from == 0) return true;
  }
  return false;
}

// A workgroup's parts, one after the other; what they are is kept in LDS: the tile loops have no registers to spare.  Pieces
// where there are few segments (whole_from), the line otherwise.
struct Line {
  Scratch scratch;
  Place place;
  Part next;
  int more, pieces;
  template <int ROWS, int KEYS>
  __device__ __forceinline__ void start(const AttendParams& p, int w) {
    const Requests<ROWS, KEYS> requests(p);
    long long upto, mine;
    const long long total = total_weight(p, requests, scratch, upto, mine);
    const long long segments = total_segments(p, requests, scratch);
    const bool by_pieces = segments < p.whole_from;  // with one more for each segment they are as many as the workgroups
    Place at{};
    Part only{};
    bool some = false;
    if (by_pieces)
      some = find_piece(p, requests, w, p.parts.borders ? share_of(p, total, p.workgroups - segments) : total + 1, scratch, only);
    else
      at = find_place(p, requests, w, total, upto, mine, scratch);
    if (threadIdx.x == 0) {
      pieces = by_pieces;
      more = some;
      next = only;
      place = at;
    }
  }
  // False: there is no further part.  Between two calls: a barrier behind the last use of the first one's part.
  template <int ROWS, int KEYS>
  __device__ __forceinline__ bool advance(const AttendParams& p, bool first, Part& part) {
    if (threadIdx.x == 0) {
      if (pieces) {
        more = more && first;
      } else {
        Place at = place;
        Part x{};
        more = next_part<ROWS, KEYS>(p, at, x);
        next = x;
        place = at;
      }
    }
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(more)) return false;
    part = stored();
    return true;
  }
  __device__ __forceinline__ Part stored() const {
    return {__builtin_amdgcn_readfirstlane(next.b), __builtin_amdgcn_readfirstlane(next.h), __builtin_amdgcn_readfirstlane(next.t),
            uniform(next.from), uniform(next.to), uniform(next.weight)};
  }
  // Where the part's rows go if it is not a whole segment: two places for each workgroup of the line, 0 for a segment that began
  // in an earlier share, 1 for one that begins in its share and goes on behind it; one for each piece.
  template <int ROWS>
  __device__ __forceinline__ long long part_rows(int w, const Part& part) const {
    return (__builtin_amdgcn_readfirstlane(pieces) ? static_cast<long long>(w) : static_cast<long long>(w) * 2 + (part.from == 0)) * ROWS;
  }
};
// The same for the join: part i of the segment that `border` of workgroup w tells of.
template <int ROWS>
__device__ __forceinline__ long long joined_rows(const Border& border, int w, int i, int H) {
  return (border.parts < 0 ? w + static_cast<long long>(i) * H : i == 0 ? (w - 1) * 2ll + 1 : (w - 1ll + i) * 2) * ROWS;
}

// Steps of a part, of the `steps` that the segment turned out to take.
__device__ __forceinline__ int steps_before(long long weight_before, long long weight, int steps) {
  return static_cast<int>(quotient(weight_before * steps, weight));
}

template <int ROWS>
__device__ __forceinline__ Tile tile_of(const Cache& c, const Part& part) {
  Tile t;
  t.b = part.b;
  fill_tile(c, t);
  t.row0 = part.t * ROWS;
  t.rows = min(t.n_new * c.G - t.row0, ROWS);
  return t;
}

}  // namespace paged
}  // namespace heatkv
