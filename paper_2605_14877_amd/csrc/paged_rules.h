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

// Steps of a share at least, measured with three requests of up to 740 keys (fp32, d = 128): 17.7 us with 8, 15.4 with 4, 17.4
// with 2.
// Where no cache is longer than WHOLE_STEPS nothing is cut: the halves would save less than the join's launch of about 4 us.
constexpr int LEAST_STEPS = 4, WHOLE_STEPS = 8;
// Requests of more query rows (new tokens x queries per kv head) than this are the 128-row kernel's.
constexpr int MANY_ROWS = 64;

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
  // Fewer segments than half of that are dealt by pieces: up to one more than shares for each.
  p.few.whole_from = 256;
  p.few.grid = 512 + 256;
  p.few.least_steps = LEAST_STEPS;
  p.few.parts = longest > WHOLE_STEPS * 32 ? 2 * 512 : 0;
  // Little more than one token for each request: taken for a decoding step, whose few padding rows are not worth a launch.
  if (bf16 && rows > MANY_ROWS && tokens > batch + 16 && (top == 0 || many_union_bytes(group, max_pages, top) <= MANY_UNION_BYTES)) {
    p.few.most_rows = p.many.least_rows = MANY_ROWS;
    p.many.workgroups = 512;
    p.many.least_steps = LEAST_STEPS;
    // Two whole segments for every share and more: nothing is cut.  Fewer: the pieces are at most one more than each
    // segment's weight is shares.
    p.many.whole_from = 1024;
    const int64_t segments = kv_heads * (rows / 128 + std::min<int64_t>(batch, rows / (MANY_ROWS + 1)));
    const int64_t pieces = p.many.workgroups + std::min<int64_t>(segments, p.many.whole_from - 1);
    const bool cut = longest > WHOLE_STEPS * 64;
    p.many.grid = cut ? std::max(segments, pieces) : segments;
    p.many.parts = cut ? static_cast<int>(pieces) : 0;
  }
  return p;
}

}  // namespace paged
}  // namespace heatkv
