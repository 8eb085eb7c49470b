// How the paged attention is launched, from sizes that the host knows: host code without HIP, so that it can be checked
// without a GPU.
#pragma once

#include <algorithm>
#include <climits>
#include <cstdint>

namespace heatkv {
namespace paged {

struct Launch {
  int workgroups = 0;              // shares that the work is cut into; 0: not launched
  int64_t grid = 0;                // workgroups launched
  int parts = 0;                   // places for parts of cut segments; 0: nothing is cut
  int whole_from = 0;              // segments from which on: few, they are dealt along a line; many, none is cut
  int least_steps = 0;             // of a share
  int least_rows = 0, most_rows = INT_MAX;  // requests by their query rows per kv head: least_rows < rows <= most_rows
};
struct Plan {
  Launch few, many;  // tiles of 16 rows and steps of 32 keys; of 128 and 64
};

// Workgroups of a launch that the join looks at: where segments are cut, no more have work than there are places for parts.  A
// larger grid is one workgroup for each segment that there may be, and from whole_from segments on none is cut.  1024 kv heads of
// 16 query heads each, 1024 requests, 8192 tokens: 2097152 workgroups, of which 1535 matter (all of them, times eight in the join,
// would be more lanes than a launch can have).
inline int join_workgroups(const Launch& l) { return static_cast<int>(std::min<int64_t>(l.grid, l.parts)); }

// Steps of a share at least, measured with three requests of up to 740 keys (fp32, d = 128): 17.7 us with 8, 15.4 with 4, 17.4
// with 2.  Where no cache is longer than WHOLE_STEPS nothing is cut: the halves would save less than the join's launch of about
// 4 us.
constexpr int LEAST_STEPS = 4, WHOLE_STEPS = 8;

// Fewer segments of 16 rows than this are dealt by pieces.  That is one wave of workgroups with an equal part for each, but
// leaves as many idle as there are segments (128: a quarter); on the line none idles, and many have the ends of two segments.
// Decoding 8, 12, 15 requests of 1000 keys over 8 heads: 15.6, 17.2, 17.8 us by pieces, 18.3, 19.3, 19.7 on the line; 16
// and 31 requests: 23.1 and 28.3 by pieces (as many as that takes), 20.2 and 26.9 on the line.
constexpr int FEW_SEGMENTS = 128;

// Requests of more query rows (new tokens x queries per kv head) than this are the 128-row kernel's, which reads their keys
// once for 128 rows, and computes for 128 as well.  16 requests of 4096 keys, 4 query rows a token: 5 tokens 98 us with 16
// rows a tile, 70 with 128, 16 tokens 174 and 83.  With chosen pages tiles of fewer tokens read fewer pages: 12 requests of
// 12000 keys, 8 tokens 75 us with 128 rows, 71 with 16; 16 tokens 87; 24 tokens 122 with 16 rows, 96 with 128.
constexpr int MANY_ROWS = 16, MANY_CHOSEN_ROWS = 64;

// More tokens than one for each request and this: before, the call is taken for a decoding step, with padding rows or a few
// tokens that are checked at once, and not worth the second kernel's launch and the longer join (up to 10 us) to look for long requests.
// One request, 24 tokens at 1000, 8000 and 32000 keys: 16, 31 and 80 us by the 16-row kernel alone, 24, 32 and 59 with both.
constexpr int FEW_TOKENS = 40, FEW_TOKENS_LONG = 16, LONG_CACHE = 16384;

// LDS of the 128-row kernel for the union of its tokens' chosen pages: a bit and a count for each word of the request's pages,
// 24 bytes for each page that may be in it.  Larger unions are left to the 16-row kernel, whose tiles have fewer tokens.
constexpr size_t MANY_LDS = 160 * 1024, MANY_UNION_BYTES = 92 * 1024;
inline size_t many_union_bytes(int group, int64_t max_pages, int64_t top) {
  const int64_t capacity = std::min<int64_t>(max_pages, std::min(128, 127 / group + 2) * top);
  return static_cast<size_t>(16 + (max_pages + 31) / 32 * 8 + capacity * 24);
}

// `top`: pages that a token reads at most, 0: all of them.
inline Plan plan_launches(bool bf16, int batch, int kv_heads, int group, int64_t tokens, int64_t max_pages, int page_size, int64_t top) {
  Plan p;
  const int64_t rows = tokens * group, longest = max_pages * page_size;
  // Two workgroups to a compute unit are resident.
  p.few.workgroups = 512;
  p.few.whole_from = FEW_SEGMENTS;
  p.few.grid = 512;
  p.few.least_steps = LEAST_STEPS;
  p.few.parts = longest > WHOLE_STEPS * 32 ? 2 * 512 : 0;
  const int many_rows = top ? MANY_CHOSEN_ROWS : MANY_ROWS;
  const int few_tokens = top == 0 && longest >= LONG_CACHE ? FEW_TOKENS_LONG : FEW_TOKENS;
  if (bf16 && rows > many_rows && tokens > batch + few_tokens && (top == 0 || many_union_bytes(group, max_pages, top) <= MANY_UNION_BYTES)) {
    p.few.most_rows = p.many.least_rows = many_rows;
    p.many.workgroups = 512;
    p.many.least_steps = LEAST_STEPS;
    // Two whole segments for every share and more: nothing is cut.  Fewer: the pieces are at most one more than each
    // segment's weight is shares.
    p.many.whole_from = 1024;
    const int64_t segments = kv_heads * (rows / 128 + std::min<int64_t>(batch, rows / (many_rows + 1)));
    const int64_t pieces = p.many.workgroups + std::min<int64_t>(segments, p.many.whole_from - 1);
    const bool cut = longest > WHOLE_STEPS * 64;
    p.many.grid = cut ? std::max(segments, pieces) : segments;
    p.many.parts = cut ? static_cast<int>(pieces) : 0;
  }
  return p;
}

}  // namespace paged
}  // namespace heatkv
