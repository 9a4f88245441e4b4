// Which entries the query tokens of a sequence see, from lengths that a device array holds.  Plain constexpr functions, used by the
// kernels and, without a GPU, by the test that looks at lengths of any value (tests/test_pages_columns.py).
#pragma once
#include <cstdint>

namespace d2o {

// Entries of a sequence that claims `len` of them: none below zero, max_len at most.
constexpr int32_t entries_of(int32_t len, int32_t max_len) { return len < 0 ? 0 : len < max_len ? len : max_len; }

// The last entry that `token` sees, one of `tokens` whose newest is entry entries - 1; -1: none.  (With entries >= 0 and tokens below 2^28 no
// difference leaves 32 bits.)
constexpr int32_t last_seen(int32_t entries, int32_t tokens, int32_t token) {
  const int32_t last = entries - tokens + token;
  return last > -1 ? last : -1;
}

// Tiles of `tile` entries that a window and the first n_sink entries show of max_len entries at most, to `columns` neighbouring tokens.
constexpr int64_t shown_tiles(int32_t max_len, int32_t window, int32_t n_sink, int32_t columns, int32_t tile) {
  const int64_t all = (int64_t(max_len) + tile - 1) / tile, shown = (int64_t(window) + n_sink + columns) / tile + 3;
  return shown < all ? shown : all;
}

}  // namespace d2o
