// Writing the 8-bit key/value cache and reading it back.
//
// Both are memory-bound (2 bytes of fp16 and 1 of codes per value) and take a
// wave to a page of one head, keys or values, with the whole page in registers:
// lane l holds 8 channels of Dp / 8 tokens.
//
// MI355X: four prompts of 1900-2048 tokens of 56 heads of 128 channels written in 66 us
// (340 MB at 5.1 TB/s; a copy reaches 5.15) and read back in 57 (6.0).  A step's single
// tokens of 64 sequences are a launch and a few latencies, 10.4 us for 40 heads: their
// values are bytes of 5120 cache lines each.
#include <math.h>

#include "ot_kv8.h"

namespace ot {
namespace detail {

constexpr int kKv8Waves = 4;  // of a workgroup, each for itself

// The sequence of slot `slot` and where its tokens start, with `at` the call's lengths
// (kLast: of the cache after the call, whose last tokens they are) or first positions.
struct Kv8Where {
  int b;  // -1: none
  Kv8Rows rows;
  int64_t start, first_slot;
};
template <bool kLast>
__device__ __forceinline__ Kv8Where kv8_where(const int32_t *__restrict__ cu,
                                              const int32_t *__restrict__ at, int B, int64_t T,
                                              int64_t slot, int lane) {
  Kv8Where w{-1, {0, 0}, 0, 0};
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int b = b0 + lane;
    int c0 = 0, c1 = 0, v = 0;
    if (b < B) {
      c0 = cu[b];
      c1 = cu[b + 1];
      v = at[b];
    }
    const int n = __popcll(__ballot(b < B && kv8_page_slot(c0, b) <= slot));
    if (n > 0) {
      c0 = __builtin_amdgcn_readlane(c0, n - 1);
      w.b = b0 + n - 1;
      w.rows = kv8_rows(c0, __builtin_amdgcn_readlane(c1, n - 1), T);
      w.start = (int64_t)__builtin_amdgcn_readlane(v, n - 1) - (kLast ? w.rows.n : 0);
      w.first_slot = kv8_page_slot(c0, w.b);
    }
    if (n < 64) break;
  }
  return w;
}

// Where a lane's u-th 8 channels (of kUnits) lie in a page.
//   keys    [64][Dp]: the page in order, so that a load takes whole rows
//   values  [Dp][64]: eight tokens of the same channels one after another, whose codes are
//           eight bytes of a channel's row then; eight lanes have 128 bytes of a token in
//           fp16 and a channel's whole row of codes.  (With four tokens to a lane, 64 bytes
//           of each, 8 sequences of 500-2000 tokens of 40 heads were read in 82 us.)
template <int DP, bool KEYS>
struct Place {
  static constexpr int kUnits = KEYS ? DP / 8 : (DP + 63) / 64 * 8;
  int token, channel;
  __device__ __forceinline__ Place(int lane, int u) {
    if constexpr (KEYS) {
      const int e = u * 64 + lane;
      token = e / (DP / 8);
      channel = e % (DP / 8) * 8;
    } else {
      token = (lane & 7) * 8 + (u & 7);
      channel = ((u >> 3) * 8 + (lane >> 3)) * 8;
    }
  }
};

// The largest bit pattern of a fp16 magnitude: NaN and infinities come last.
__device__ __forceinline__ uint32_t most_bits(uint32_t most, v4u x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = x[i] & 0x7fff7fffu;
    most = max(most, max(w & 0xffffu, w >> 16));
  }
  return most;
}

// A code as its byte in the low bits: rne(x inv) clipped to +-127, plus 128.  The
// sum with 1.5 2^23 + 128 rounds to a whole number (its last place is 1; 128 is
// even, so ties go the same way) whose low bits are the byte.
__device__ __forceinline__ uint32_t code_byte(float x, float inv) {
  const float v = __builtin_amdgcn_fmed3f(x * inv, -127.f, 127.f) + 12583040.f;
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
  const uint32_t cd = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
  return ab | cd;
}
__device__ __forceinline__ float half_at(v4u x, int i) {
  return half_bits_to_float((uint16_t)(x[i >> 1] >> (16 * (i & 1))));
}

// A byte's code divided by 2^k, rounded to nearest even.
__device__ __forceinline__ uint32_t shrink_bytes(uint32_t w, float f) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float c = (float)(int)((w >> (8 * i)) & 0xffu) - 128.f;
    out |= (uint32_t)(int)(rintf(c * f) + 128.f) << (8 * i);
  }
  return out;
}

// The scale of a page and head is the largest magnitude of the tokens that it is first
// written with over 127; where a later token does not fit, it grows by the power of two
// that makes it fit and the codes that are there are divided by that: their error stays
// below one step of the scale, as 1/2 + 1/4 + 1/8 + ... of it, however often it grows.
//
// Takes the page's scale to new tokens of the largest magnitude with the bits `most` (of
// any lane's), from place lo on, and the codes before them with it; returns what turns a
// value into a code.
template <int DP, bool KEYS>
__device__ __forceinline__ float rescale_page(uint32_t most, bool has_old, int lo, int lane,
                                              uint8_t *__restrict__ codes, float *__restrict__ scale) {
  const float old = has_old ? *scale : 0.f;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
  const float a = half_bits_to_float((uint16_t)most);
  float s = a / 127.f;
  int k = 0;
  if (old > 0.f) {
    const float fits = 127.5f * old;
    if (a > fits) {  // the exponents' difference, one more where the fraction is larger
      const uint32_t ab = __builtin_bit_cast(uint32_t, a), fb = __builtin_bit_cast(uint32_t, fits);
      k = (int)(ab >> 23) - (int)(fb >> 23) + ((ab & 0x7fffffu) > (fb & 0x7fffffu));
    }
    s = ldexpf(old, k);
  }
  if (most >= 0x7c00u || old != old) s = __builtin_nanf("");
  if (k > 0) {
    // earlier tokens' codes: 16 bytes of one token (keys) or of 16 tokens (values)
    const float f = ldexpf(1.f, -k);
#pragma unroll 4
    for (int u = 0; u < DP / 16; ++u) {
      const int at = (u * 64 + lane) * 16;
      if ((KEYS ? at / DP : at % kKv8Page) < lo) {
        v4u w = *reinterpret_cast<const v4u *>(codes + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = shrink_bytes(w[i], f);
        *reinterpret_cast<v4u *>(codes + at) = w;
      }
    }
    __threadfence_block();  // a word with both gets its new codes last
  }
  if (lane == 0) *scale = s;
  return s > 0.f ? 1.f / s : 0.f;
}

// A few tokens, as decode and drafts write: a lane has two channels (four past 128) of
// each, so that a load or store takes a whole row.
constexpr int kFewTokens = 8;
template <int DP, bool KEYS>
__device__ __forceinline__ void append_few(const uint16_t *__restrict__ x, int64_t ld, int D, int lane,
                                           int lo, int count, bool has_old, bool there,
                                           uint8_t *__restrict__ codes, float *__restrict__ scale) {
  constexpr int kPairs = (DP + 127) / 128;
  uint32_t r[kFewTokens][kPairs], most = 0;
#pragma unroll
  for (int i = 0; i < kFewTokens; ++i)
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const int c = 128 * k + 2 * lane;
      r[i][k] = i < count && c < D ? *reinterpret_cast<const uint32_t *>(x + i * ld + c) : 0u;
    }
  if (!there) return;
#pragma unroll
  for (int i = 0; i < kFewTokens; ++i)
#pragma unroll
    for (int k = 0; k < kPairs; ++k) most = max(most, max(r[i][k] & 0x7fffu, r[i][k] >> 16 & 0x7fffu));
  const float inv = rescale_page<DP, KEYS>(most, has_old, lo, lane, codes, scale);
#pragma unroll
  for (int i = 0; i < kFewTokens; ++i) {
    if (i >= count) break;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const int c = 128 * k + 2 * lane;
      if (c >= D) continue;
      const uint32_t b0 = code_byte(half_bits_to_float((uint16_t)r[i][k]), inv);
      const uint32_t b1 = code_byte(half_bits_to_float((uint16_t)(r[i][k] >> 16)), inv);
      if constexpr (KEYS) {
        *reinterpret_cast<uint16_t *>(codes + (lo + i) * DP + c) = (uint16_t)((b0 & 0xffu) | b1 << 8);
      } else {
        codes[c * kKv8Page + lo + i] = (uint8_t)b0;
        codes[(c + 1) * kKv8Page + lo + i] = (uint8_t)b1;
      }
    }
  }
}

// Any number of tokens, in the page's own order.
template <int DP, bool KEYS>
__device__ __forceinline__ void append_page(const uint16_t *__restrict__ x, int64_t ld, int D, int lane,
                                            int lo, int hi, bool has_old, uint8_t *__restrict__ codes,
                                            float *__restrict__ scale) {
  using At = Place<DP, KEYS>;
  constexpr int kUnits = At::kUnits;
  v4u r[kUnits];
  uint32_t most = 0;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const At at(lane, u);
    const int t = at.token, c = at.channel;
    r[u] = v4u{0u, 0u, 0u, 0u};
    if (t >= lo && t < hi && c < D)
      r[u] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(x + (t - lo) * ld + c));
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) most = most_bits(most, r[u]);
  const float inv = rescale_page<DP, KEYS>(most, has_old, lo, lane, codes, scale);
  if constexpr (KEYS) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const At at(lane, u);
      uint32_t b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = code_byte(half_at(r[u], i), inv);
      if (at.token >= lo && at.token < hi)
        *reinterpret_cast<v2u *>(codes + at.token * DP + at.channel) =
            v2u{low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7])};
    }
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; u += 8) {
      const At at(lane, u);
      const int t = at.token;
      if (t + 8 > lo && t < hi && at.channel < DP) {
        const bool whole = t >= lo && t + 8 <= hi;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t b[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = code_byte(half_at(r[u + j], i), inv);
          uint8_t *p = codes + (at.channel + i) * kKv8Page + t;
          if (whole) {
            *reinterpret_cast<v2u *>(p) =
                v2u{low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7])};
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (t + j >= lo && t + j < hi) p[j] = (uint8_t)b[j];
          }
        }
      }
    }
  }
}

template <int DP>
__global__ __launch_bounds__(64 * kKv8Waves) void kv8_append_kernel(
    const uint16_t *__restrict__ k, int64_t ldk, const uint16_t *__restrict__ v, int64_t ldv,
    int64_t T, int B, int H, int D, const int32_t *__restrict__ cu,
    const int32_t *__restrict__ kv_len, Kv8Cache cache) {
  const int lane = threadIdx.x;
  const int unit = blockIdx.y * kKv8Waves + threadIdx.y;
  if (unit >= 2 * H) return;
  const int64_t slot = blockIdx.x;
  const Kv8Where w = kv8_where<true>(cu, kv_len, B, T, slot, lane);
  if (w.b < 0) return;
  const Kv8Touch at = kv8_touch(w.start, w.rows.n, slot - w.first_slot);
  if (at.lo >= at.hi || at.col < 0) return;
  int64_t page = kv8_page(cache.table, w.b, at.col, cache.max_pages, cache.num_pages);
  const bool there = page >= 0;
  if (!there) page = 0;
  const int64_t row = w.rows.row0 + (at.col * kKv8Page + at.lo - w.start);
  const int h = unit >> 1, count = at.hi - at.lo;
  const int64_t ph = page * H + h;
  const bool old = w.start > at.col * kKv8Page;
  const bool keys = (unit & 1) == 0;
  const uint16_t *x = keys ? k + row * ldk + h * D : v + row * ldv + h * D;
  const int64_t ld = keys ? ldk : ldv;
  uint8_t *codes = (keys ? cache.Kc : cache.Vc) + ph * (DP * kKv8Page);
  float *scale = (keys ? cache.Ks : cache.Vs) + ph;
  if (count <= kFewTokens) {  // loads ahead of the page's number
    if (keys)
      append_few<DP, true>(x, ld, D, lane, at.lo, count, old, there, codes, scale);
    else
      append_few<DP, false>(x, ld, D, lane, at.lo, count, old, there, codes, scale);
  } else if (there) {
    if (keys)
      append_page<DP, true>(x, ld, D, lane, at.lo, at.hi, old, codes, scale);
    else
      append_page<DP, false>(x, ld, D, lane, at.lo, at.hi, old, codes, scale);
  }
}

__device__ __forceinline__ uint32_t value_pair(uint32_t a, uint32_t b, float s) {
  const uint32_t x = float_to_half_bits(((float)(int)a - 128.f) * s);
  const uint32_t y = float_to_half_bits(((float)(int)b - 128.f) * s);
  return x | y << 16;
}

template <int DP>
__global__ __launch_bounds__(64 * kKv8Waves) void kv8_read_kernel(
    Kv8Cache cache, int H, int D, const int32_t *__restrict__ cu,
    const int32_t *__restrict__ start, int64_t T, int B, uint16_t *__restrict__ k,
    uint16_t *__restrict__ v) {
  const int lane = threadIdx.x;
  const int unit = blockIdx.y * kKv8Waves + threadIdx.y;
  if (unit >= 2 * H) return;
  const int64_t slot = blockIdx.x;
  const Kv8Where w = kv8_where<false>(cu, start, B, T, slot, lane);
  if (w.b < 0) return;
  const Kv8Touch at = kv8_touch(w.start, w.rows.n, slot - w.first_slot);
  if (at.lo >= at.hi) return;
  int64_t page = kv8_page(cache.table, w.b, at.col, cache.max_pages, cache.num_pages);
  const bool none = page < 0;
  if (none) page = 0;
  const int64_t row = w.rows.row0 + (at.col * kKv8Page + at.lo - w.start);
  const int h = unit >> 1;
  const int64_t ph = page * H + h;
  if ((unit & 1) == 0) {
    const float s = none ? __builtin_nanf("") : cache.Ks[ph];
    const uint8_t *p = cache.Kc + ph * (DP * kKv8Page);
    uint16_t *out = k + (row * H + h) * D;
    constexpr int kAtOnce = DP / 8 < 16 ? DP / 8 : DP / 16;
#pragma unroll 1
    for (int u0 = 0; u0 < DP / 8; u0 += kAtOnce) {
      // loads have no condition, or each would wait for the one before: lanes without a
      // token take another's
      v2u w[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const Place<DP, true> place(lane, u0 + u);
        w[u] = *reinterpret_cast<const v2u *>(p + min(max(place.token, at.lo), at.hi - 1) * DP + place.channel);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const Place<DP, true> place(lane, u0 + u);
        const int t = place.token, c = place.channel;
        if (t < at.lo || t >= at.hi || c >= D) continue;
        v4u y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = w[u][i >> 1] >> (16 * (i & 1));
          y[i] = value_pair(x & 0xffu, x >> 8 & 0xffu, s);
        }
        __builtin_nontemporal_store(y, reinterpret_cast<v4u *>(out + (int64_t)(t - at.lo) * H * D + c));
      }
    }
  } else {
    const float s = none ? __builtin_nanf("") : cache.Vs[ph];
    const uint8_t *p = cache.Vc + ph * (DP * kKv8Page);
    uint16_t *out = v + (row * H + h) * D;
    constexpr int kGroups = Place<DP, false>::kUnits / 8, kAtOnce = kGroups == 3 ? 3 : kGroups < 2 ? 1 : 2;
    static_assert(kGroups % kAtOnce == 0, "whole groups");
#pragma unroll 1
    for (int g0 = 0; g0 < kGroups; g0 += kAtOnce) {
      v2u w[kAtOnce][8];
#pragma unroll
      for (int g = 0; g < kAtOnce; ++g) {
        const Place<DP, false> place(lane, 8 * (g0 + g));
        const int t = min(max(place.token, at.lo & ~7), (at.hi - 1) & ~7), c = min(place.channel, DP - 8);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          w[g][i] = *reinterpret_cast<const v2u *>(p + (c + i) * kKv8Page + t);
      }
#pragma unroll
      for (int g = 0; g < kAtOnce; ++g) {
        const Place<DP, false> place(lane, 8 * (g0 + g));
        const int t = place.token, c = place.channel;
        if (t + 8 <= at.lo || t >= at.hi || c >= D) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (t + j < at.lo || t + j >= at.hi) continue;
          v4u y;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y[i] = value_pair(w[g][2 * i][j >> 2] >> (8 * (j & 3)) & 0xffu,
                              w[g][2 * i + 1][j >> 2] >> (8 * (j & 3)) & 0xffu, s);
          __builtin_nontemporal_store(y, reinterpret_cast<v4u *>(out + (int64_t)(t + j - at.lo) * H * D + c));
        }
      }
    }
  }
}

}  // namespace detail

#define OT_KV8_WIDTH(dp, call)          \
  switch (dp) {                         \
    case 64: call(64); break;           \
    case 96: call(96); break;           \
    case 128: call(128); break;         \
    case 192: call(192); break;         \
    default: call(256); break;          \
  }

hipError_t launch_kv8_append(const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv,
                             int64_t T, int64_t B, int64_t H, int64_t D, const int32_t *cu,
                             const int32_t *kv_len, const Kv8Cache &cache, hipStream_t st) {
  const dim3 grid((unsigned)kv8_page_slots(T, B),
                  (unsigned)((2 * H + detail::kKv8Waves - 1) / detail::kKv8Waves));
  const dim3 block(64, detail::kKv8Waves);
#define OT_CALL(dp)                                                                            \
  detail::kv8_append_kernel<dp><<<grid, block, 0, st>>>(k, ldk, v, ldv, T, (int)B, (int)H, (int)D, cu, \
                                                        kv_len, cache)
  OT_KV8_WIDTH(kv8_width(D), OT_CALL)
#undef OT_CALL
  return hipGetLastError();
}

hipError_t launch_kv8_read(const Kv8Cache &cache, int64_t H, int64_t D, const int32_t *cu,
                           const int32_t *start, int64_t T, int64_t B, uint16_t *k, uint16_t *v,
                           hipStream_t st) {
  const dim3 grid((unsigned)kv8_page_slots(T, B),
                  (unsigned)((2 * H + detail::kKv8Waves - 1) / detail::kKv8Waves));
  const dim3 block(64, detail::kKv8Waves);
#define OT_CALL(dp)                                                                            \
  detail::kv8_read_kernel<dp><<<grid, block, 0, st>>>(cache, (int)H, (int)D, cu, start, T, (int)B, k, v)
  OT_KV8_WIDTH(kv8_width(D), OT_CALL)
#undef OT_CALL
  return hipGetLastError();
}

}  // namespace ot
