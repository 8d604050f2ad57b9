// Device helpers that the MX4 linear's tile kernels share: the matrix step, the
// tile schedule and the epilogue.
#pragma once

#include "ot_mx4.h"

namespace ot {
namespace detail {

// The token and channel tile of this workgroup: each XCD a contiguous range of
// tiles, walked in groups of 8 token tiles, so that concurrent tiles share
// operand rows in the XCD's L2 (as the int8 prefill).
// Several of these per tile (parts of K) follow one another as whole launches.
struct TilePlace {
  int tm, tn, part;
  __device__ __forceinline__ TilePlace(int tiles_m, int tiles_n, bool parts) {
    constexpr int kGroupM = 8;
    const int nwg = gridDim.x, bid = blockIdx.x;
    const int xcd = bid & 7, local = bid >> 3;
    const int per = nwg >> 3, rem = nwg & 7;
    int lid = (xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per) + local;
    part = 0;
    if (parts) {
      part = lid / (tiles_m * tiles_n);
      lid %= tiles_m * tiles_n;
    }
    const int group_size = kGroupM * tiles_n;
    const int first_m = (lid / group_size) * kGroupM;
    const int gm = min(tiles_m - first_m, kGroupM);
    tm = first_m + (lid % group_size) % gm;
    tn = (lid % group_size) / gm;
  }
};

__device__ __forceinline__ int swz_mx4(int r) { return (r & 7) ^ ((r >> 3) & 1); }

template <int kStep>
__device__ __forceinline__ v16f mfma_mx4(v4i a, v4i b, v16f c, int ea, int eb) {
  const v8i a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const v8i b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, kStep, ea, kStep, eb);
}

template <int V>
struct IntC {
  static constexpr int value = V;
};

// Bias, fp16 and whole token rows out, through the wave's part of the idle LDS:
// the block of kFN x kFM 32x32 tiles from channel nw0 and token mw0 on.  Every
// wave of the workgroup is done with its LDS.
template <int kFN, int kFM>
__device__ __forceinline__ void mx4_epilogue(uint8_t *smem, const v16f (&acc)[kFN][kFM],
                                             const float *__restrict__ bp, int M, int N,
                                             uint16_t *__restrict__ Y, int nw0, int64_t mw0,
                                             int wave, int lane) {
  constexpr int kTN = 32 * kFN, kTM = 32 * kFM;
  const int fr = lane & 31, fh = lane >> 5;
  // Lane l of a 32x32 block holds token l mod 32 and, in registers 4j..4j+3,
  // channels 8j + 4 (l / 32) .. +3.  The wave's kTM token rows of kTN channels
  // are staged with the 8-byte unit u of row r at unit u ^ h(r), which spreads
  // the lanes of a write over the banks.
  constexpr int kUnits = kTN / 4;
  constexpr int kSwz = kUnits % 16 == 0 ? 16 : 8;
  constexpr int kCpr = kTN / 8;
  static_assert(kUnits % kSwz == 0, "the swizzle permutes whole groups of units");
  auto stage_swz = [](int r) { return kSwz == 16 ? (r & 15) : ((r >> 1) & 7); };
  uint16_t *tile = reinterpret_cast<uint16_t *>(smem) + wave * (kTM * kTN);
#pragma unroll
  for (int f = 0; f < kFN; ++f)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int nl = f * 32 + 8 * j + 4 * fh, n = nw0 + nl;
      float4 b4 = make_float4(0.f, 0.f, 0.f, 0.f);
      if (n + 3 < N) {
        b4 = *reinterpret_cast<const float4 *>(bp + n);
      } else {
        if (n + 0 < N) b4.x = bp[n + 0];
        if (n + 1 < N) b4.y = bp[n + 1];
        if (n + 2 < N) b4.z = bp[n + 2];
      }
#pragma unroll
      for (int g = 0; g < kFM; ++g) {
        const int r = g * 32 + fr;
        uint2 h;
        h.x = (uint32_t)float_to_half_bits(acc[f][g][4 * j] + b4.x) |
              ((uint32_t)float_to_half_bits(acc[f][g][4 * j + 1] + b4.y) << 16);
        h.y = (uint32_t)float_to_half_bits(acc[f][g][4 * j + 2] + b4.z) |
              ((uint32_t)float_to_half_bits(acc[f][g][4 * j + 3] + b4.w) << 16);
        *reinterpret_cast<uint2 *>(tile + r * kTN + 4 * ((nl >> 2) ^ stage_swz(r))) = h;
      }
    }
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_wave_barrier();
  if ((N & 7) == 0) {
#pragma unroll 2
    for (int c0 = 0; c0 < kTM * kCpr; c0 += 64) {
      const int c = c0 + lane;
      const int r = c / kCpr, cc = c % kCpr;
      const int x = stage_swz(r);
      uint4 v = *reinterpret_cast<const uint4 *>(tile + r * kTN + (cc ^ (x >> 1)) * 8);
      if (x & 1) {  // the two 8-byte units of the pair are stored swapped
        const uint32_t t0 = v.x, t1 = v.y;
        v.x = v.z; v.y = v.w; v.z = t0; v.w = t1;
      }
      const int64_t m = mw0 + r;
      const int n = nw0 + cc * 8;
      if (m < M && n < N) *reinterpret_cast<uint4 *>(Y + m * (int64_t)N + n) = v;
    }
    return;
  }
  // Token rows that are not 16-byte aligned: a word (two channels) to a lane, 32
  // channels of four rows at a time; the words of a row that starts at an odd
  // halfword begin one channel earlier, so that its first and last channels stand
  // alone.  On MI355X 6241 tokens x 660, K = 3328 take 18.0 us, x 661 19.5 and x 664
  // 17.2; with 16 bytes to a lane, stored by halfwords, 23.1.
  auto at = [&](int r, int e) { return tile + r * kTN + 4 * ((e >> 2) ^ stage_swz(r)) + (e & 3); };
  const int q = lane & 15, r0 = lane >> 4;
  const int rows = (int)(M - mw0 < kTM ? M - mw0 : kTM);
  auto words = [&](auto odd) {
    constexpr int kOdd = decltype(odd)::value;
    const int p = kOdd ? (int)((mw0 + r0) & 1) : 0;
#pragma unroll
    for (int j = 0; j < kTN / 32; ++j) {
      const int e = 32 * j + 2 * q - p, n = nw0 + e;
      const bool lo = e >= 0 && n < N, hi = n + 1 < N;
      uint16_t *dst = Y + (mw0 + r0) * (int64_t)N + n;
#pragma unroll 4
      for (int r = r0; r < rows; r += 4, dst += 4 * (int64_t)N) {
        if constexpr (kOdd == 0) {
          if (lo) *reinterpret_cast<uint32_t *>(dst) = *reinterpret_cast<const uint32_t *>(at(r, e));
        } else {
          const uint32_t v0 = *at(r, max(e, 0)), v1 = *at(r, e + 1);
          if (lo && hi) *reinterpret_cast<uint32_t *>(dst) = v0 | v1 << 16;
          else if (lo) dst[0] = (uint16_t)v0;
          else if (hi) dst[1] = (uint16_t)v1;
          if (j == 0 && e < 0 && nw0 + kTN - 1 < N) dst[kTN] = *at(r, kTN - 1);
        }
      }
    }
  };
  if (N & 1) words(IntC<1>{});
  else words(IntC<0>{});
}

}  // namespace detail
}  // namespace ot
