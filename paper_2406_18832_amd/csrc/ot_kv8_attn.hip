// Attention over the 8-bit cache: which kernel a call takes, and its workspace.
#include <stdio.h>

#include "ot_kv8_attn.h"

namespace ot {
namespace {

// Up to so many query rows to a key head and sequence the kernel for few rows runs.
constexpr int64_t kFewRows = 32;
// Pages to an item, at least, and pages of a sequence up to which it is not split: a
// second launch takes as long as a workgroup's waves take for so many.
constexpr int kLeastPages = 4, kWholePages = 16;

bool few_rows(int64_t G, int64_t max_q) { return max_q * G <= kFewRows; }

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

}  // namespace

// Fewer than 2^32 work-items: tiles of 128 rows, and up to wanted + B items, all heads,
// 256 threads each; rows of a key head below 2^30.
bool attn_kv8_fits(int64_t T, int64_t B, int64_t Hq, int64_t Hkv) {
  const int64_t G = Hq / Hkv, limit = (int64_t(1) << 32) / 256;
  return T * G < (int64_t(1) << 30) && kv8_tile_slots(T * G, B, 128) * Hkv < limit &&
         (B + 4096) * Hkv < limit && (Hkv * kFewRows / 4 + 1) * B < limit;
}

size_t attn_kv8_workspace_bytes(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D,
                                int64_t max_q) {
  Kv8Split s;
  return plan_split(B, Hq, Hkv, D, max_q, s);
}

hipError_t launch_attn_kv8(const Kv8Attn &a, void *workspace, hipStream_t st) {
  if (!few_rows(a.Hq / a.Hkv, a.max_q)) return launch_kv8_tiles(a, st);
  Kv8Split s;
  const size_t bytes = plan_split(a.B, a.Hq, a.Hkv, a.D, a.max_q, s);
  if (workspace == nullptr || bytes == 0 || a.cache.max_pages <= kWholePages) {
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
  Kv8Split s;
  const size_t bytes = plan_split(B, Hq, Hkv, D, max_q, s);
  if (!few_rows(Hq / Hkv, max_q))
    snprintf(buf, len, "tiles 256");
  else if (workspace && bytes != 0)
    snprintf(buf, len, "few %d rows, %lld items", max_q * (Hq / Hkv) <= 16 ? 16 : 32, (long long)s.items);
  else
    snprintf(buf, len, "few %d rows", max_q * (Hq / Hkv) <= 16 ? 16 : 32);
}

}  // namespace ot
