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

// Where no segment can be cut, pieces are whole segments, one to a workgroup, and further workgroups for those that are more than are
// resident; on the line a workgroup has up to four in its share, one after the other, and other workgroups have none.  Every workgroup
// looks for its own, which takes longer from one request to a lane on.  Decoding with up to 240 keys, 8 heads, 16 and 64 requests of
// different lengths, 4-bit rows: 8.9 and 10.5 us by pieces, 18.0 and 22.9 on the line; of equal lengths, bf16: 9.7 and 15.8, 10.2 and
// 16.1; 128 requests: 22.5 and 42.6, of equal lengths 31.1 and 26.6.  A prompt of 240 tokens, fp32: 12.4 and 21.3, eight of them: 49.6
// and 60.8.  Where the 128-row kernel is launched as well there may be nothing to do for the grid of a workgroup to a segment (eight
// prompts of 240 tokens: 18.0 us, 13.4 without).
constexpr int WHOLE_SEGMENTS = 2560, WHOLE_BATCH = 64;

// Requests of more query rows (new tokens x queries per kv head) than this are the 128-row kernel's, which reads their keys
// once for 128 rows, and computes for 128 as well.  16 requests of 4096 keys, 4 query rows a token: 5 tokens 98 us with 16
// rows a tile, 70 with 128, 16 tokens 174 and 83.  With chosen pages tiles of fewer tokens read fewer pages: 12 requests of
// 12000 keys, 8 tokens 75 us with 128 rows, 71 with 16; 16 tokens 87; 24 tokens 122 with 16 rows, 96 with 128.
constexpr int MANY_ROWS = 16, MANY_CHOSEN_ROWS = 64;

// More tokens than one for each request and this: before, the call is taken for a decoding step, with padding rows or a few
// tokens that are checked at once, and not worth the second kernel's workgroups and the longer join (3 us) to look for long requests.
// One request, 24 tokens at 1000, 8000 and 32000 keys: 16, 29 and 80 us by the 16-row kernel alone, 19, 26 and 48 with both.
constexpr int FEW_TOKENS = 40, FEW_TOKENS_LONG = 16, LONG_CACHE = 16384;

// Where both kernels have work, one launch has the workgroups of both.  Those of many rows come first, and what few requests of few rows
// there may be falls into the gaps at their end; over all pages, from more requests than this on, those of few rows come first, which read
// memory while the others compute.  Many rows first, few rows first, two launches, bf16, d = 128: 8 requests that decode over 1000 keys and
// two prompts of 300 tokens 27, 31, 34 us, 32 and two 39, 42, 48, 48 and two 52, 52, 59; 32 requests over 9000 keys and 1000 new tokens
// over 2000: 283, 260, 285, 48 and those 382, 356, 386; whole scales of 8 requests, 4-bit rows, d = 64: 51, 56, 59.
constexpr int FEW_FIRST = 32;

// LDS of a compute unit, and of the 128-row kernel for the union of its tokens' chosen pages: a bit and a count for each word of the
// request's pages, 24 bytes for each page that may be in it.  Larger unions are left to the 16-row kernel, whose tiles have fewer tokens.
constexpr size_t MANY_LDS = 160 * 1024, MANY_UNION_BYTES = 92 * 1024;
inline size_t many_union_bytes(int group, int64_t max_pages, int64_t top) {
  const int64_t capacity = std::min<int64_t>(max_pages, std::min(128, 127 / group + 2) * top);
  return static_cast<size_t>(16 + (max_pages + 31) / 32 * 8 + capacity * 24);
}

// With chosen pages those of many rows come first: they take longer then, and the others read little.  64 requests that decode and two
// chunks of 1000 tokens, 32 pages of 64 keys for each token, many first, few first, two launches: bf16, d = 128 and 64: 332, 344, 356 us
// and 205, 271, 249; 8 bits: 289, 320, 329 and 219, 235, 242; 4 bits: 265, 280, 286 and 182, 221, 209.  Where the tokens of a chunk all
// choose the same pages few first is faster at d = 128: 64 requests and 500 tokens, bf16 91 and 85, 4 bits 66 and 62 (d = 64: 53 and 57, 48
// and 45).
// Where the union's LDS leaves room for one workgroup on a compute unit, few rows in the same launch would have but one as well:
// they get a launch of their own.  64 requests of 200000 keys and a chunk of 500 tokens, 80 pages each: 4 bits, d = 128 and 64: 172, 172,
// 146 us and 142, 142, 122; 8 bits: 188, 184, 180 and 145, 145, 128; bf16, d = 64: 162, 156, 156.  Rows of 256 bytes are read as fast by
// one workgroup to a unit (242, 228, 241).  200 requests of 64000 keys, four chunks, 26 pages: 4 bits, d = 128: 287, 287, 255; bf16: 357,
// 346, 352.
enum class FewRows { BEHIND, IN_FRONT, APART };
inline FewRows place_of_few(int batch, bool chosen, size_t lds, int row_bytes) {
  if (!chosen) return batch > FEW_FIRST ? FewRows::IN_FRONT : FewRows::BEHIND;
  if (2 * lds <= MANY_LDS) return FewRows::BEHIND;
  return batch > FEW_FIRST && row_bytes >= 256 ? FewRows::IN_FRONT : FewRows::APART;
}

// `top`: pages that a token reads at most, 0: all of them.
inline Plan plan_launches(bool bf16, int batch, int kv_heads, int group, int64_t tokens, int64_t max_pages, int page_size, int64_t top) {
  Plan p;
  const int64_t rows = tokens * group, longest = max_pages * page_size;
  // Two workgroups to a compute unit are resident.  Of the 128-row kernel at d = 64, bf16 and 4-bit rows, three are; as many shares cut keys
  // that need not be.  512, 640, 768 shares, 4-bit rows: whole scales of 8 requests 53, 61, 60 us, 4 x 700 tokens over as many keys
  // before them 55, 55, 66, 1000 tokens over 4096 68, 72, 72, 2 x 2048 tokens 231 with all; bf16 the same.
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
  if (!p.few.parts && batch <= WHOLE_BATCH) {
    const int64_t segments = kv_heads * (rows / 16 + std::min<int64_t>(batch, tokens));
    if (!p.many.workgroups && segments <= WHOLE_SEGMENTS) p.few.grid = std::max(segments, p.few.grid);
    p.few.whole_from = static_cast<int>(p.few.grid) + 1;
  }
  return p;
}

}  // namespace paged
}  // namespace heatkv
