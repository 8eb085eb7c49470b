// How the paged attention launches are cut, from sizes that the host knows: host code without HIP, so that it can be checked
// without a GPU.
#pragma once

#include <algorithm>
#include <cstdint>

namespace heatkv {
namespace paged {

constexpr int MANY_ROWS = 64;  // the long kernel's requests have more query rows per kv head (paged.h: LONG_ROWS)

struct Split {
  int few;   // workgroups per tile of 16 rows
  int many;  // workgroups per tile of 128 rows; 0: no request is the long kernel's
};

// `longest`: keys that a request can have at most; `chosen`: keys that a token reads at most (0: all).
// Lengths are on the device, so this goes by what the launch could need: workgroups enough for every compute unit to have
// four (two of the long kernel), a part no shorter than 256 keys.
inline Split plan_splits(bool bf16, int batch, int kv_heads, int group, int64_t tokens, int64_t longest, int64_t chosen) {
  const int64_t rows = tokens * group;
  // As many tokens as requests or fewer: taken for single tokens.  Otherwise any request may have many rows.
  const bool may_be_long = bf16 && chosen == 0 && tokens > batch && rows > MANY_ROWS;
  auto cut = [&](int64_t tiles, int64_t wanted, int64_t keys) {
    const int64_t parts = (wanted + tiles * kv_heads - 1) / (tiles * kv_heads);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({parts, (keys + 255) / 256, 64})));
  };
  const int64_t few_tiles = tokens <= batch ? std::max<int64_t>(tokens, 1) : std::max<int64_t>((rows + 15) / 16, 1);
  Split s;
  s.few = cut(may_be_long ? std::max<int64_t>(batch, 1) : few_tiles, 1024, chosen ? std::min(chosen * std::min<int64_t>(16, tokens), longest) : longest);
  s.many = may_be_long ? cut((rows + 127) / 128, 512, longest) : 0;
  return s;
}

}  // namespace paged
}  // namespace heatkv
