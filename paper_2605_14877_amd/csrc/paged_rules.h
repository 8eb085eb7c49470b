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
  int whole_from = INT_MAX;        // segments from which on a workgroup takes one, uncut
  int least_steps = 0;             // of a share
  int least_rows = 0, most_rows = INT_MAX;  // requests by their query rows per kv head: least_rows < rows <= most_rows
  bool join = false;               // segments may be cut
};
struct Plan {
  Launch few, many;  // tiles of 16 rows and steps of 32 keys; of 128 and 64
};

// Requests of more query rows (new tokens x queries per kv head) than this are the 128-row kernel's.
constexpr int MANY_ROWS = 64;

// `longest`: keys that a request can have at most; `chosen`: keys that a token reads at most (0: all of them).
inline Plan plan_launches(bool bf16, int batch, int kv_heads, int group, int64_t tokens, int64_t longest, int64_t chosen) {
  Plan p;
  const int64_t rows = tokens * group;
  p.few.workgroups = 512;
  p.few.grid = 512;
  p.few.least_steps = 8;
  p.few.join = longest > 8 * 32;
  if (bf16 && chosen == 0 && rows > MANY_ROWS) {
    p.few.most_rows = p.many.least_rows = MANY_ROWS;
    p.many.workgroups = 512;
    p.many.least_steps = 8;
    // Two whole segments and more for every share: dealt as workgroups come free.
    p.many.whole_from = 1024;
    const int64_t most = kv_heads * (rows / 128 + std::min<int64_t>(batch, rows / (MANY_ROWS + 1)));
    p.many.grid = most >= p.many.whole_from ? most : p.many.workgroups;
    p.many.join = longest > 8 * 64;
  }
  return p;
}

}  // namespace paged
}  // namespace heatkv
