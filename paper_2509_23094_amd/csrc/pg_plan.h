// Whole-number arithmetic of the paged attention's plans, for host and device alike (constexpr functions; no HIP in this file).
#pragma once
#include <stdint.h>

namespace d2c {

struct PgSpan { int row0, m; };
// The rows of the batch between two row starts, whatever these hold: each is taken into [0, n_rows] before the difference, which a start of -2^31 would
// otherwise carry past 32 bits; none where they do not ascend.
constexpr PgSpan pg_span(int lo, int hi, int n_rows) {
  const int first = lo < 0 ? 0 : lo < n_rows ? lo : n_rows, end = hi < 0 ? 0 : hi < n_rows ? hi : n_rows;
  return PgSpan{first, end > first ? end - first : 0};
}

// How many of `tiles` stay whole: a share that is a little above 1 where all do (see make_plan), so that from 2^20 tiles on the product would pass them.
constexpr int pg_whole(int tiles, float share) {
  const int n = (int)((float)tiles * share);
  return n < tiles ? n : tiles;
}

// Workgroup wg of `count` in a round that goes backwards: by eights, which stay on their XCD; those that fill no eight keep their place.
constexpr int pg_backwards(int wg, int count) { return wg < count / 8 * 8 ? (count / 8 - 1 - wg / 8) * 8 + wg % 8 : wg; }

}  // namespace d2c
