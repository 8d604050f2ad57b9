// The 8-bit key/value cache: its format in registers and its launchers.
//
// A page holds 64 tokens of every head: codes of 8 bits and one scale, for keys
// and for values.  A byte b stands for the code b - 128.  Bytes past a page's
// tokens and past D channels can be anything: every byte is a finite code, and
// what they meet in a product is 0.
#pragma once

#include "ot_common.h"
#include "ot_kv8_index.h"

namespace ot {

// Widths of a page's rows: the template of every kernel.
constexpr int kKv8Widths[] = {64, 96, 128, 192, 256};
inline int kv8_width(int64_t D) {
  for (int w : kKv8Widths)
    if (D <= w) return w;
  return 0;
}

struct Kv8Cache {
  uint8_t *Kc, *Vc;  // [pages][H][64][Dp], [pages][H][Dp][64]
  float *Ks, *Vs;    // [pages][H]
  const int32_t *table;
  int64_t max_pages, num_pages;
};

struct Kv8Attn {
  const uint16_t *q;
  int64_t ldq;
  int T, B, Hq, Hkv, D;
  int max_q;  // queries of a sequence past these are left out (few rows)
  const int32_t *cu, *kv_len;
  Kv8Cache cache;
  float scale;
  int causal;
  int64_t window;
  uint16_t *Y;
  float *lse;  // or nullptr
};

hipError_t launch_kv8_append(const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv,
                             int64_t T, int64_t B, int64_t H, int64_t D, const int32_t *cu,
                             const int32_t *kv_len, const Kv8Cache &cache, hipStream_t st);
hipError_t launch_kv8_read(const Kv8Cache &cache, int64_t H, int64_t D, const int32_t *cu,
                           const int32_t *start, int64_t T, int64_t B, uint16_t *k, uint16_t *v,
                           hipStream_t st);
// workspace: nullptr, or attn_kv8_workspace_bytes of the same sizes.
hipError_t launch_attn_kv8(const Kv8Attn &a, void *workspace, hipStream_t st);
// The launches of these sizes stay within the limits of a grid.
bool attn_kv8_fits(int64_t T, int64_t B, int64_t Hq, int64_t Hkv);
size_t attn_kv8_workspace_bytes(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D,
                                int64_t max_q);
void describe_attn_kv8(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_q,
                       bool workspace, char *buf, size_t len);

namespace detail {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Four bytes of the cache as their codes in fp16, exactly: the byte b under the
// high byte 0x64 is the fp16 value 1024 + b, and 1024 + b - 1152 = b - 128.
__device__ __forceinline__ v4h kv8_halves(uint32_t w) {
  const v2h bias = {(_Float16)-1152.f, (_Float16)-1152.f};
  const v2h lo = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + bias;
  const v2h hi = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + bias;
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
}
__device__ __forceinline__ v8h kv8_halves(uint32_t a, uint32_t b) {
  return __builtin_shufflevector(kv8_halves(a), kv8_halves(b), 0, 1, 2, 3, 4, 5, 6, 7);
}

// The sequence that takes slot `at`: the number of sequences whose first slot lies
// at or before it, less one (-1 for none).  Every lane of the wave takes part.
template <class F>
__device__ __forceinline__ int kv8_find(int B, int lane, int64_t at, F first_slot) {
  int count = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int b = b0 + lane;
    const int c = __popcll(__ballot(b < B && first_slot(b) <= at));
    count += c;
    if (c < 64) break;
  }
  return count - 1;
}

}  // namespace detail
}  // namespace ot
