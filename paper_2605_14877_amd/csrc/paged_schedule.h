// How a launch's work is dealt to workgroups when the lengths are on the device.
//
// A segment is a tile of query rows of a request and kv head, and has a weight, about proportional to the keys that it walks
// over.  All segments lie on one line: requests in order, of each the kv heads, of each the tiles.  Workgroup w takes the
// stretch [w share, (w + 1) share) of it, so any mix of lengths is dealt evenly, with a grid that depends on nothing that the
// host does not know.  A segment that crosses from one share into another is computed in parts (its steps in proportion to
// the weight on either side), which a second launch joins in order; light segments are not cut, they belong to the
// workgroup that they begin in.
//
// Every workgroup finds its place by a scan over the requests (two rounds of loads, a block scan: about 2 us).
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

struct Place {
  long long pos, stop, share;  // on the line; pos >= stop: nothing (more) to do
  int b, h, t;                 // the segment at pos
  long long off;               // pos in it
  Load load;                   // of request b
};
struct Scratch {  // LDS
  long long sums[4], more_sums[4], first;
  int b;
};

template <int ROWS, int KEYS>
__device__ __forceinline__ Load request_load(const AttendParams& p, int b) {
  return load_of<ROWS, KEYS>(p, uniform_load(p.c.q_start, b), uniform_load(p.c.q_start, b + 1), uniform_load(p.c.lens, b));
}

// Inclusive sums over the 256 lanes of a workgroup, and the total in `all`; `sums`: LDS, free at the next barrier but one.
__device__ __forceinline__ long long block_scan(long long v, long long (&sums)[4], long long& all) {
  const int tid = threadIdx.x, lane = tid & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long long u = __shfl_up(v, d, 64);
    if (lane >= d) v += u;
  }
  if (lane == 63) sums[tid >> 6] = v;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long x = sums[i];
    if (i < (tid >> 6)) v += x;
    all += x;
  }
  all = uniform(all);
  return v;
}
// The request that holds position `at` of a line on which request b takes cost(b), and where on the line it begins.  By all
// lanes; `upto`: block_scan of the costs of this lane's requests, `mine`.
template <class Cost>
__device__ __forceinline__ int find_request_at(long long at, int batch, long long upto, long long mine, const Cost& cost,
                                               Scratch& scratch, long long& first) {
  const int per = (batch + 255) / 256;
  if (at < upto && at >= upto - mine) {  // one lane
    long long x = upto - mine;
    for (int i = 0; i < per; ++i) {
      const int b = threadIdx.x * per + i;
      const long long n = b < batch ? cost(b) : 0;
      if (at < x + n) {
        scratch.first = x;
        scratch.b = b;
        break;
      }
      x += n;
    }
  }
  __syncthreads();
  first = uniform(scratch.first);
  return __builtin_amdgcn_readfirstlane(scratch.b);
}
template <class Cost>
__device__ __forceinline__ long long own_cost(int batch, const Cost& cost) {  // of this lane's requests
  const int per = (batch + 255) / 256;
  long long mine = 0;
  for (int i = 0; i < per; ++i)
    if (static_cast<int>(threadIdx.x) * per + i < batch) mine += cost(threadIdx.x * per + i);
  return mine;
}

// The place of workgroup w, by all of its 256 lanes.
template <int ROWS, int KEYS>
__device__ __forceinline__ Place find_place(const AttendParams& p, int w, Scratch& scratch) {
  const Cache& c = p.c;
  auto cost = [&](int b) {
    const Load l = load_of<ROWS, KEYS>(p, c.q_start[b], c.q_start[b + 1], c.lens[b]);
    return l.upto(l.tiles) * c.H;
  };
  const long long mine = own_cost(c.batch, cost);
  long long total;
  const long long upto = block_scan(mine, scratch.sums, total);
  Place at{};
  at.share = max((total + p.workgroups - 1) / p.workgroups, static_cast<long long>(p.least_weight));
  at.pos = w * at.share;
  at.stop = min(at.pos + at.share, total);
  if (at.pos >= total) return at;
  long long first;
  at.b = find_request_at(at.pos, c.batch, upto, mine, cost, scratch, first);
  at.load = request_load<ROWS, KEYS>(p, at.b);
  const long long rel = at.pos - first, per_head = at.load.upto(at.load.tiles);
  at.h = static_cast<int>(rel / per_head);
  const long long in_head = rel - at.h * per_head;
  int below = 0, above = at.load.tiles;  // the last tile that begins at in_head or before
  while (above - below > 1) {
    const int mid = (below + above) >> 1;
    (at.load.upto(mid) <= in_head ? below : above) = mid;
  }
  at.t = below;
  at.off = in_head - at.load.upto(below);
  return at;
}

// The part of the segment at pos that is this workgroup's; advances the place behind it.
struct Part {
  int b, h, t;
  long long from, to, weight;  // of the segment's weight; the whole segment: from == 0, to == weight
};
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

// What the join has to know about the border between shares w - 1 and w: written by workgroup w, before its first part.
// parts 0: no segment is cut there, or it was cut at an earlier border already.
__device__ __forceinline__ void write_border(const AttendParams& p, const Place& at, int w) {
  if (!p.borders || threadIdx.x != 0) return;
  Border x{at.b, at.h, at.t, 0};
  if (at.pos < at.stop && at.off > 0 && at.off <= at.share) {
    const long long weight = at.load.weight(at.t);
    if (weight > p.cut_from) x.parts = 1 + static_cast<int>((weight - at.off + at.share - 1) / at.share);
  }
  p.borders[w] = x;
}

// The other way to deal, for large tiles: a workgroup takes one piece, and pieces come as workgroups become free.  A segment
// is one piece where there are segments enough to fill the chip evenly (whole_from), otherwise as many as its request's mean
// weight is shares (`workgroups` of them, none lighter than least_weight).  Parts are fewer than on the line, and the tile
// loop needs no registers for a place on it.  The last tiles come first: with a causal limit they are the heaviest.
// Pieces of a segment lie H workgroups apart.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool find_piece(const AttendParams& p, int w, Scratch& scratch, Part& part) {
  const Cache& c = p.c;
  auto load = [&](int b) { return load_of<ROWS, KEYS>(p, c.q_start[b], c.q_start[b + 1], c.lens[b]); };
  auto weight = [&](int b) {
    const Load l = load(b);
    return l.upto(l.tiles) * c.H;
  };
  auto segments = [&](int b) { return static_cast<long long>(load(b).tiles) * c.H; };
  long long total, count;
  block_scan(own_cost(c.batch, weight), scratch.sums, total);
  block_scan(own_cost(c.batch, segments), scratch.more_sums, count);
  const long long share = count >= p.whole_from || !p.borders ? total + 1 : max((total + p.workgroups - 1) / p.workgroups, static_cast<long long>(p.least_weight));
  auto cuts = [&](const Load& l) {
    return l.tiles ? static_cast<int>((l.upto(l.tiles) / l.tiles + share - 1) / share) : 0;
  };
  auto pieces = [&](int b) {
    const Load l = load(b);
    return static_cast<long long>(l.tiles) * cuts(l) * c.H;
  };
  const long long mine = own_cost(c.batch, pieces);
  long long all, first;
  const long long upto = block_scan(mine, scratch.sums, all);
  if (p.borders && threadIdx.x == 0) p.borders[w].parts = 0;
  if (w >= all) return false;
  part.b = find_request_at(w, c.batch, upto, mine, pieces, scratch, first);
  const Load l = request_load<ROWS, KEYS>(p, part.b);
  const int n = cuts(l), rel = static_cast<int>(w - first), i = rel / c.H, tile = i / n;
  part.h = rel - i * c.H;
  part.t = l.tiles - 1 - tile;
  part.from = i - tile * n;
  part.to = part.from + 1;
  part.weight = n;
  if (p.borders && threadIdx.x == 0 && n > 1 && part.from == 0) p.borders[w] = Border{part.b, part.h, part.t, n};
  return true;
}

// A workgroup's place on the line and the part at hand, in LDS: the tile loops have no registers to spare for them.
struct Line {
  Scratch scratch;
  Place place;
  Part next;
  int more;
  template <int ROWS, int KEYS>
  __device__ __forceinline__ void start(const AttendParams& p, int w) {
    const Place at = find_place<ROWS, KEYS>(p, w, scratch);
    write_border(p, at, w);
    if (threadIdx.x == 0) place = at;
  }
  // False: there is no further part.  Between two calls: a barrier behind the last use of the first one's part.
  template <int ROWS, int KEYS>
  __device__ __forceinline__ bool advance(const AttendParams& p, Part& part) {
    if (threadIdx.x == 0) {
      Place at = place;
      Part x{};
      more = next_part<ROWS, KEYS>(p, at, x);
      next = x;
      place = at;
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
};

// Steps of a part, of the `steps` that the segment turned out to take.
__device__ __forceinline__ int steps_before(long long weight_before, long long weight, int steps) {
  return static_cast<int>(weight_before * steps / weight);
}

// Where a workgroup puts its parts: 0 a segment that began in an earlier share, 1 one that begins in its share and goes on
// behind it; ROWS rows each.
template <int ROWS>
__device__ __forceinline__ long long part_rows(int w, bool begins) {
  return (static_cast<long long>(w) * 2 + (begins ? 1 : 0)) * ROWS;
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
