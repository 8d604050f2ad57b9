// Attention over the 8-bit cache: which kernel a call takes, and its workspace.
#include <stdio.h>

#include "ot_kv8_attn.h"

namespace ot {
namespace {

// Pages to an item, at least, and pages of a sequence up to which it is not split: a
// second launch takes as long as a workgroup's waves take for so many (of tiles that leave
// less than half of the device idle: a few per cent, which pays from kManyPages on; 1941
// tokens of 24 heads over 9000-48000 keys, 364 tiles for 512 workgroups, 485 us against
// 1058).  More tiles than the device takes at a time are not split (8192 tokens of 12 heads
// of 64 channels, 768 tiles: 161 us against 200).  Both
// rules go by the number of tiles, not by how much longer than an even share the longest is,
// which costs a causal prompt of about as many tiles as run at a time: 4096 tokens of 8 heads
// of 256 channels, 256 tiles of 1 to 64 pages on 256 CUs, take 186 us, as long as without a
// mask (190).
constexpr int kLeastPages = 4, kWholePages = 16, kManyPages = 128;
// Parts of a tile's pages, at most.
constexpr int64_t kMostParts = 64;
// Windows below this take tiles of 128 rows.
constexpr int64_t kWideWindow = 1500;

bool few_rows(int64_t G, int64_t max_q) { return max_q * G <= kFewRows; }

// Pages that `tokens` of a sequence one after another see, at most.
int64_t most_pages(const Kv8Attn &a, int64_t tokens) {
  const int64_t all = a.cache.max_pages;
  return a.window > 0 ? kv8_min(all, (a.window + tokens) / kKv8Page + 2) : all;
}

// How a call of few rows is split, and the bytes that takes (0: not at all).
size_t plan_split(int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_q, Kv8Split &s) {
  const int64_t G = Hq / Hkv;
  s = Kv8Split{};
  s.items = B;
  s.rows = max_q * G;
  s.least = kLeastPages;
  if (!few_rows(G, max_q)) return 0;
  // as many workgroups as run at a time
  const int dp = kv8_width(D), tiles = kv8_decode_tiles(dp, s.rows);
  const int64_t per_item = Hkv * ((s.rows + 16 * tiles - 1) / (16 * tiles));
  const int64_t wanted = (int64_t)device_cus() * kv8_decode_waves(dp, tiles) / per_item;
  s.wanted = (int)(wanted > 0 ? wanted : 1);
  s.items = s.wanted + B;
  const int64_t rows = s.items * Hkv * s.rows;
  return (size_t)(B + (B & 1)) * sizeof(int2) + (size_t)(rows + (rows & 1)) * 2 * sizeof(float) +
         (size_t)rows * dp * sizeof(float);
}

// Tiles of many rows: their size and how many parts their pages are shared in.  128 rows
// take two workgroups to a CU, of which one works while the other starts or ends.  256 rows,
// one to a CU, take less time for a page, which pays where a tile has many: for 128
// channels, some 3000 rows and more to a sequence, and a tile for most CUs.  MI355X, 256
// against 128 rows: an 8192-token prompt of 72 heads 1165 us against 1268, 4096 tokens of
// 8 x 4 heads 149 against 177, 2 x 1024 tokens of 8 x 4 heads in a window of 4096 147 against
// 166; 2048 tokens of 40 heads 72 against 67, 32 prompts of 512 tokens 279 against 232; with
// 64 channels 8192 tokens of 12 heads 186 against 164, with 96 up to 3 % less.  With 192
// channels the stages of a page leave LDS for one workgroup of either: 12 prompts of 1300
// tokens of 3 x 5 heads of 144 channels 155 against 240 (150 in products of 160 channels).
// With 256 they leave registers for one wave to a SIMD, and 128 rows.
// A small window leaves a tile few pages: 4096 tokens of 40 heads in one of 512 tokens 134 us
// against 97 (6 pieces of 700-1000 tokens of 8 x 4 heads: 100 against 89; of 1024 tokens 142
// against 139, of 2048 228 against 240).
// Bytes of the workspace (0: none).
size_t plan_tiles(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int &rows, Kv8Parts &p) {
  const int64_t G = Hq / Hkv, cus = device_cus();
  const int dp = kv8_width(D);
  rows = dp == 192 || (dp == 128 && T * G >= 3000 * B && T * G * Hkv / 256 >= cus * 3 / 4) ? 256 : 128;
  p = Kv8Parts{};
  p.parts = 1;
  p.least = 4;
  p.rows = T * Hq;
  const int64_t tiles = (T * G / rows + (B + 1) / 2) * Hkv;  // half a tile of each sequence is empty
  p.groups = (int)(rows == 128 && dp <= 128 ? 2 * cus : cus);
  if (tiles > p.groups) return 0;
  const int64_t parts = kv8_min(4 * p.groups / tiles, kMostParts);
  p.parts = (int)parts;
  p.whole = 2 * tiles <= p.groups ? kWholePages : kManyPages;
  const int64_t all = p.rows + (p.rows & 1);
  return sizeof(float) * (size_t)(2 * all + 2 * parts * all + parts * p.rows * dp);
}

}  // namespace

// Fewer than 2^32 work-items: T G / 128 + B tiles of 128 rows by 256 threads, or
// T G / 256 + B of 256 rows by 512 (several parts only where there are few), up to
// wanted + B items by 256, of all heads; rows of a key head below 2^30.
bool attn_kv8_fits(int64_t T, int64_t B, int64_t Hq, int64_t Hkv) {
  const int64_t G = Hq / Hkv, limit = (int64_t(1) << 32) / 256;
  return T * G < (int64_t(1) << 30) && (T * G / 128 + 2 * B) * Hkv < limit &&
         (B + 4096) * Hkv < limit && (Hkv * kFewRows / 4 + 1) * B < limit && T * Hq / 4 < limit;
}

size_t attn_kv8_workspace_bytes(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D,
                                int64_t max_q) {
  Kv8Split s;
  Kv8Parts p;
  int rows;
  return few_rows(Hq / Hkv, max_q) ? plan_split(B, Hq, Hkv, D, max_q, s)
                                   : plan_tiles(T, B, Hq, Hkv, D, rows, p);
}

hipError_t launch_attn_kv8(const Kv8Attn &a, void *workspace, hipStream_t st) {
  if (!few_rows(a.Hq / a.Hkv, a.max_q)) {
    Kv8Parts p;
    int rows;
    const size_t bytes = plan_tiles(a.T, a.B, a.Hq, a.Hkv, a.D, rows, p);
    if (a.window > 0 && a.window < kWideWindow && kv8_width(a.D) == 128) rows = 128;
    if (workspace == nullptr || bytes == 0 || most_pages(a, rows) <= p.whole) {
      p.parts = 1;
      return launch_kv8_tiles(a, rows, p, st);
    }
    const int64_t all = p.rows + (p.rows & 1);
    p.counts = static_cast<int *>(workspace);
    p.m = reinterpret_cast<float *>(p.counts + 2 * all);
    p.l = p.m + p.parts * all;
    p.o = p.l + p.parts * all;
    const hipError_t e = launch_kv8_tiles(a, rows, p, st);
    return e != hipSuccess ? e : launch_kv8_join(a, p, st);
  }
  Kv8Split s;
  const size_t bytes = plan_split(a.B, a.Hq, a.Hkv, a.D, a.max_q, s);
  if (workspace == nullptr || bytes == 0 || most_pages(a, a.max_q) <= kWholePages) {
    s.wanted = 0;
    s.items = a.B;
    return launch_kv8_decode(a, s, st);
  }
  const int64_t rows = s.items * a.Hkv * s.rows;
  s.spans = static_cast<int2 *>(workspace);
  s.m = reinterpret_cast<float *>(s.spans + a.B + (a.B & 1));
  s.l = s.m + rows + (rows & 1);
  s.o = s.l + rows + (rows & 1);
  const hipError_t e = launch_kv8_decode(a, s, st);
  return e != hipSuccess ? e : launch_kv8_combine(a, s, st);
}

void describe_attn_kv8(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_q,
                       bool workspace, char *buf, size_t len) {
  if (!few_rows(Hq / Hkv, max_q)) {
    Kv8Parts p;
    int rows;
    plan_tiles(T, B, Hq, Hkv, D, rows, p);
    if (workspace && p.parts > 1)
      snprintf(buf, len, "tiles %d, %d parts", rows, p.parts);
    else
      snprintf(buf, len, "tiles %d", rows);
    return;
  }
  Kv8Split s;
  const size_t bytes = plan_split(B, Hq, Hkv, D, max_q, s);
  const int at_once = 16 * kv8_decode_tiles(kv8_width(D), s.rows);
  if (workspace && bytes != 0)
    snprintf(buf, len, "few %d rows, %lld items", at_once, (long long)s.items);
  else
    snprintf(buf, len, "few %d rows", at_once);
}

}  // namespace ot
