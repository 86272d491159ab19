// rows_cost.cpp -- the counting of kv_rows_cost.h for a whole call, in 32 bits as the kernel does and in 64.
#include "kv_rows_cost.h"

extern "C" int rows_total(int64_t n, const int32_t* pos, const int32_t* members, int32_t n_heads, int32_t heads,
                          int32_t tiles, int32_t tile_rows, int step_log, int64_t max_tokens, int32_t window,
                          int prefixes, uint64_t* total, int64_t* least) {
  int64_t rows = 0;
  for (int64_t i = 0; i < n; ++i) rows += members[i];
  const p2p::RowsScale s = p2p::rows_scale(n, rows, n_heads, heads, tiles, tile_rows, step_log, max_tokens);
  const int64_t group = n_heads / heads, unit = (int64_t)tiles * tile_rows;
  *total = 0, *least = INT64_MAX;
  int same = 1;
  for (int64_t i = 0; i < n; ++i) {
    const p2p::RowsCost c = prefixes ? p2p::RowsCost::of_prefix(0, pos[i], s, step_log)
                                     : p2p::RowsCost::of_prompt(pos[i], window, s, step_log);
    const uint32_t count = (uint32_t)((members[i] * group + unit - 1) / unit);
    uint64_t before = 0;
    for (uint32_t j = 0; j <= count; j += count > 5000 && j + 5000 < count ? count / 5000 : 1) {  // (some of many)
      const uint64_t x = c.of<uint64_t>(j);
      same &= x == c.of(j);
      if (j > 0 && (int64_t)(x - before) < *least) *least = (int64_t)(x - before);
      before = x;
    }
    *total += before * heads;
  }
  return same;
}
