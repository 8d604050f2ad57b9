// Which tokens and pages a workgroup of the 8-bit cache's kernels takes: plain
// arithmetic, for the device and (in tests) for the host.
//
// The lengths are on the device, where the host cannot check them, so every
// index that comes from memory is brought into its range here: a row offset
// into 0..T, a page number that is none of the cache's to -1 (what the callers
// do with it is theirs to say), a length to what the table has pages for.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define OT_HD __host__ __device__ __forceinline__
#else
#define OT_HD inline
#endif

namespace ot {

constexpr int kKv8Page = 64;  // tokens

OT_HD int64_t kv8_min(int64_t a, int64_t b) { return a < b ? a : b; }
OT_HD int64_t kv8_max(int64_t a, int64_t b) { return a > b ? a : b; }

// Rows [row0, row0 + n) of a batch of T rows are sequence b's.
struct Kv8Rows {
  int row0, n;
};
OT_HD Kv8Rows kv8_rows(int cu0, int cu1, int64_t T) {
  const int64_t a = kv8_min(kv8_max(cu0, 0), T), b = kv8_min(kv8_max(cu1, a), T);
  return {(int)a, (int)(b - a)};
}

// Sequences take slots, so that a launch whose size depends on T and B alone has
// one for each of their units (tiles of `unit` rows, or pages).  The first slot of
// the sequence whose rows start at `row`:
//   tiles  floor(row / unit) + b: ceil(n / unit) units fit before the next one's
//   pages  floor(row / 64) + 2 b: n tokens from any position on touch at most
//          floor((n + 62) / 64) + 1 <= floor(n / 64) + 2 pages
OT_HD int64_t kv8_tile_slot(int64_t row, int64_t b, int unit) { return row / unit + b; }
OT_HD int64_t kv8_page_slot(int64_t row, int64_t b) { return row / kKv8Page + 2 * b; }
// and the number of slots of T rows.
OT_HD int64_t kv8_tile_slots(int64_t T, int64_t B, int unit) { return T / unit + B; }
OT_HD int64_t kv8_page_slots(int64_t T, int64_t B) { return T / kKv8Page + 2 * B; }

// The j-th page that tokens [start, start + n) of a sequence touch: the sequence's
// page number `col` (below 0 for a start below 0) and their places [lo, hi) in it;
// lo >= hi where there is no such page (for any j: offsets that fall can find a slot up to
// 2^25 and more before their sequence's first, whose distance in tokens passes 32 bits).
struct Kv8Touch {
  int64_t col;
  int lo, hi;
};
OT_HD Kv8Touch kv8_touch(int64_t start, int64_t n, int64_t j) {
  const int64_t first = start >= 0 ? start / kKv8Page : -((-start + kKv8Page - 1) / kKv8Page);
  const int64_t col = first + j, at = col * kKv8Page;
  return {col, (int)kv8_min(kv8_max(start, at) - at, kKv8Page),
          (int)kv8_max(kv8_min(start + n, at + kKv8Page) - at, -1)};
}

// A page of the cache, -1 for one that it does not have.
OT_HD int64_t kv8_page(const int32_t *table, int64_t b, int64_t col, int64_t max_pages,
                       int64_t num_pages) {
  if (col < 0 || col >= max_pages) return -1;
  const int64_t page = table[b * max_pages + col];
  return page >= 0 && page < num_pages ? page : -1;
}

// Pages [p0, p1) hold every key that queries i0 .. i0 + rows - 1 of a sequence see,
// which has n of them and len keys (as many as the table has pages for).  Query i
// stands at position len - n + i; it sees keys up to there (causal), and of those
// the last `window` (0: all).  Empty where none of them sees a key.
struct Kv8Span {
  int p0, p1;
};
OT_HD Kv8Span kv8_span(int64_t len, int64_t n, int64_t i0, int64_t rows, int causal,
                       int64_t window) {
  const int64_t end = causal ? kv8_min(len, len - n + i0 + rows) : len;
  const int64_t begin = window > 0 ? kv8_max(0, len - n + i0 - window + 1) : 0;
  if (end <= begin) return {0, 0};
  return {(int)(begin / kKv8Page), (int)((end + kKv8Page - 1) / kKv8Page)};
}
OT_HD int64_t kv8_len(int64_t len, int64_t max_pages) {
  return kv8_min(kv8_max(len, 0), max_pages * kKv8Page);
}

}  // namespace ot
