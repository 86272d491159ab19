// kv_rows_cost.h -- how the schedule of kv_rows.cuh counts its work: what its host code and the kernel have to agree on.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define P2P_BOTH __host__ __device__ __forceinline__
#else
#define P2P_BOTH inline
#endif

namespace p2p {

constexpr uint32_t kRowsSet = 2;  // steps that a unit counts for beyond its own
constexpr int kSlopeLog = 16;

// How a call's work is counted: in units of 2^shift steps, where a tile of rows (a unit) is slope / 2^kSlopeLog steps of
// tokens long.
struct RowsScale {
  int32_t shift;
  uint32_t slope;
};

// What the first j tiles of an item count for: each kRowsSet for itself and about its steps.  Any rising function would
// do, as long as all CTAs take the same and a tile counts for more than kRowsSet: a share that ends kRowsSet after a
// unit's begin has none of its steps.
struct RowsCost {
  uint32_t base, most;     // the first tile's; what none passes
  uint32_t slope, rising;  // each has slope more than the one before, for so many tiles
  int32_t shift;

  // Tiles that see tokens first .. shared - 1 alike.
  static P2P_BOTH RowsCost of_prefix(int32_t first, int32_t shared, RowsScale s, int step_log) {
    const int32_t steps = (((shared - 1) >> step_log) - (first >> step_log) + 1) >> s.shift;
    return {(steps > 1 ? steps : 1) + kRowsSet, 0, 0, ~0u, s.shift};
  }
  // Tiles of consecutive tokens from pos on, each of which sees those up to itself, the last `window` of them (0: all).
  static P2P_BOTH RowsCost of_prompt(int32_t pos, int32_t window, RowsScale s, int step_log) {
    const uint32_t steps = ((uint32_t)(pos >> step_log) + 1) >> s.shift;
    RowsCost c = {(steps > 1 ? steps : 1) + kRowsSet, 0, s.slope, ~0u, s.shift};
    if (window) {
      const uint32_t most = ((uint32_t)(window >> step_log) + (s.slope >> kSlopeLog) + 2) >> s.shift;
      c.most = (most > 1 ? most : 1) + kRowsSet;
      const uint32_t rise = c.most > c.base ? (c.most - c.base) << s.shift : 0;
      c.rising = ((rise < 1u << 15 ? rise : 1u << 15) << kSlopeLog) / s.slope;
    }
    return c;
  }
  // (T: 32 bits, which rows_scale sees to.)
  template <class T = uint32_t>
  P2P_BOTH T of(uint32_t j) const {
    const uint32_t r = j < rising ? j : rising;
    return (T)r * base + (T)((uint64_t)r * (r + 1) * slope >> (kSlopeLog + 1 + shift)) + (T)(j - r) * most;
  }
};

// For a call with n_rows rows of n_heads query heads each, in up to `items` items (none without a row), over a cache of
// `heads` heads whose sequences have up to max_tokens tokens (the window is less, or 0): `tiles` row tiles of tile_rows
// rows (104 at least) in a unit, steps of 2^step_log tokens.  The counts of all units are less than 2^32: an item of m
// tokens after pos has T = m * group / unit + 1 tiles at most, which are T * slope <= m / step + 2 steps long, so that
// none counts for more than kRowsSet + 1 + ((pos + m) / step + 3) / 2^shift.
inline RowsScale rows_scale(int64_t items, int64_t n_rows, int32_t n_heads, int32_t heads, int32_t tiles,
                            int32_t tile_rows, int step_log, int64_t max_tokens) {
  const int64_t group = n_heads / heads, unit = (int64_t)tiles * tile_rows;
  RowsScale s = {0, (uint32_t)((unit << kSlopeLog) / (group << step_log))};
  const double units = (double)(items < n_rows ? items : n_rows) * heads + (double)n_rows * n_heads / unit;
  const double steps = (double)(max_tokens >> step_log) + 4;
  while (units * (kRowsSet + 2 + steps / (double)(1ll << s.shift)) > 4e9) ++s.shift;
  return s;
}

}  // namespace p2p
