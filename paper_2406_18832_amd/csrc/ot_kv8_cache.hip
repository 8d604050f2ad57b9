// Writing the 8-bit key/value cache and reading it back.
//
// Both are memory-bound (2 bytes of fp16 and 1 of codes per value) and take a
// wave to a page of one head, keys or values, with the whole page in registers:
// lane l holds 8 channels of Dp / 8 tokens.
#include <math.h>

#include "ot_kv8.h"

namespace ot {
namespace detail {

constexpr int kKv8Waves = 4;  // of a workgroup, each for itself

// Where a lane's u-th 8 channels (of Dp / 8) lie in a page.
//   keys    [64][Dp]: the page in order, so that a load takes whole rows
//   values  [Dp][64]: four tokens of the same channels one after another, whose
//           codes are words of four tokens then, and 16 lanes write 64 bytes of a
//           channel's row
template <int DP, bool KEYS>
__device__ __forceinline__ void page_place(int lane, int u, int &token, int &channel) {
  if constexpr (KEYS) {
    const int e = u * 64 + lane;
    token = e / (DP / 8);
    channel = e % (DP / 8) * 8;
  } else {
    token = (lane & 15) * 4 + (u & 3);
    channel = ((u >> 2) * 4 + (lane >> 4)) * 8;
  }
}

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

// New tokens' codes.  The scale of a page and head is the largest magnitude of
// the tokens that it is first written with over 127; where a later token does not
// fit, it grows by the power of two that makes it fit and the codes that are
// there are divided by that: their error stays below one step of the scale, as
// 1/2 + 1/4 + 1/8 + ... of it, however often it grows.
template <int DP, bool KEYS>
__device__ __forceinline__ void append_page(const uint16_t *__restrict__ x, int64_t ld, int D,
                                            int lane, int64_t row, int lo, int hi, bool has_old,
                                            uint8_t *__restrict__ codes, float *__restrict__ scale) {
  constexpr int kUnits = DP / 8;
  v4u r[kUnits];
  uint32_t most = 0;
  const float old = has_old ? *scale : 0.f;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    int t, c;
    page_place<DP, KEYS>(lane, u, t, c);
    r[u] = v4u{0u, 0u, 0u, 0u};
    if (t >= lo && t < hi && c < D)
      r[u] = *reinterpret_cast<const v4u *>(x + (row + t - lo) * ld + c);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) most = most_bits(most, r[u]);
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
  const float inv = s > 0.f ? 1.f / s : 0.f;
  if (lane == 0) *scale = s;
  if constexpr (KEYS) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      int t, c;
      page_place<DP, KEYS>(lane, u, t, c);
      uint32_t b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = code_byte(half_at(r[u], i), inv);
      if (t >= lo && t < hi)
        *reinterpret_cast<v2u *>(codes + t * DP + c) =
            v2u{low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7])};
    }
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; u += 4) {
      int t, c;
      page_place<DP, KEYS>(lane, u, t, c);
      if (t + 4 > lo && t < hi) {
        const bool whole = t >= lo && t + 4 <= hi;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t b[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = code_byte(half_at(r[u + j], i), inv);
          uint8_t *p = codes + (c + i) * kKv8Page + t;
          if (whole) {
            *reinterpret_cast<uint32_t *>(p) = low_bytes(b[0], b[1], b[2], b[3]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
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
  const int b = kv8_find(B, lane, slot, [&](int i) { return kv8_page_slot(cu[i], i); });
  if (b < 0) return;
  const Kv8Rows rows = kv8_rows(cu[b], cu[b + 1], T);
  const int64_t start = (int64_t)kv_len[b] - rows.n;
  const Kv8Touch at = kv8_touch(start, rows.n, slot - kv8_page_slot(cu[b], b));
  if (at.lo >= at.hi) return;
  const int64_t page = kv8_page(cache.table, b, at.col, cache.max_pages, cache.num_pages);
  if (page < 0) return;
  const int64_t row = rows.row0 + (at.col * kKv8Page + at.lo - start);
  const int h = unit >> 1;
  const int64_t ph = page * H + h;
  const bool old = start > at.col * kKv8Page;
  if ((unit & 1) == 0)
    append_page<DP, true>(k + h * D, ldk, D, lane, row, at.lo, at.hi, old,
                          cache.Kc + ph * (DP * kKv8Page), cache.Ks + ph);
  else
    append_page<DP, false>(v + h * D, ldv, D, lane, row, at.lo, at.hi, old,
                           cache.Vc + ph * (DP * kKv8Page), cache.Vs + ph);
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
  const int b = kv8_find(B, lane, slot, [&](int i) { return kv8_page_slot(cu[i], i); });
  if (b < 0) return;
  const Kv8Rows rows = kv8_rows(cu[b], cu[b + 1], T);
  const int64_t first = start[b];
  const Kv8Touch at = kv8_touch(first, rows.n, slot - kv8_page_slot(cu[b], b));
  if (at.lo >= at.hi) return;
  int64_t page = kv8_page(cache.table, b, at.col, cache.max_pages, cache.num_pages);
  const bool none = page < 0;
  if (none) page = 0;
  const int64_t row = rows.row0 + (at.col * kKv8Page + at.lo - first);
  const int h = unit >> 1;
  const int64_t ph = page * H + h;
  if ((unit & 1) == 0) {
    const float s = none ? __builtin_nanf("") : cache.Ks[ph];
    const uint8_t *p = cache.Kc + ph * (DP * kKv8Page);
    uint16_t *out = k + (row * H + h) * D;
#pragma unroll 4
    for (int u = 0; u < DP / 8; ++u) {
      int t, c;
      page_place<DP, true>(lane, u, t, c);
      if (t < at.lo || t >= at.hi || c >= D) continue;
      const v2u w = *reinterpret_cast<const v2u *>(p + t * DP + c);
      v4u y;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = w[i >> 1] >> (16 * (i & 1));
        y[i] = value_pair(x & 0xffu, x >> 8 & 0xffu, s);
      }
      *reinterpret_cast<v4u *>(out + (int64_t)(t - at.lo) * H * D + c) = y;
    }
  } else {
    const float s = none ? __builtin_nanf("") : cache.Vs[ph];
    const uint8_t *p = cache.Vc + ph * (DP * kKv8Page);
    uint16_t *out = v + (row * H + h) * D;
#pragma unroll 2
    for (int u = 0; u < DP / 8; u += 4) {
      int t, c;
      page_place<DP, false>(lane, u, t, c);
      if (t + 4 <= at.lo || t >= at.hi || c >= D) continue;
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = *reinterpret_cast<const uint32_t *>(p + (c + i) * kKv8Page + t);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (t + j < at.lo || t + j >= at.hi) continue;
        v4u y;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = value_pair(w[2 * i] >> (8 * j) & 0xffu, w[2 * i + 1] >> (8 * j) & 0xffu, s);
        *reinterpret_cast<v4u *>(out + (int64_t)(t + j - at.lo) * H * D + c) = y;
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
