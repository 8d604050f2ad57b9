// Streaming MX4 weights past a few tokens: the inner loop that the decode
// linear and the mixture-of-experts layer share.
//
// Weights are read once, straight into registers in operand order, so what
// bounds these kernels is how many bytes are in flight.  A wave takes 16-row
// units (half of a packed 32-row block) by whole K tiles of 256 channels; the
// waves of a workgroup take the K tiles of the same rows in turn and their sums
// meet in LDS.  kDepth K tiles of a wave are in flight at a time.
//
// v_mfma_scale_f32_16x16x128_f8f6f4: lane l holds row l mod 16 and, with
// q = l / 16, one block of 32 channels and its scale byte.  Instruction p of a K
// tile's two gives lane group q block 4h + s with h = q mod 2 and s = 2p + q / 2,
// so that a lane's scales lie in one word (half h of the row's eight) and, once
// that word is shifted down by q / 2 bytes, instruction p picks byte 2p.
#pragma once

#include "ot_mx4.h"

namespace ot {
namespace detail {

template <int kByte>
__device__ __forceinline__ v4f mfma_mx4_16(v4i a, v4i b, v4f c, uint32_t ea, uint32_t eb) {
  const v8i a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const v8i b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, kByte, (int)ea, kByte,
                                                          (int)eb);
}

// A wave's view of packed weights: the rows of RB 16-row units from unit u0 on.
template <int RB>
struct Mx4Rows {
  const uint8_t *codes[RB];  // this lane's first 16 bytes of unit i, K tile 0
  const uint8_t *scales[RB];
  int64_t scale_step;        // bytes from a K tile's scales to the next one's

  // units: 16-row units of the whole matrix (the last one stands in past it)
  __device__ __forceinline__ void aim(const uint8_t *Wp, int64_t blocks, int64_t tiles, int64_t u0,
                                      int lane) {
    const int r = lane & 15, q = lane >> 4;
    const uint8_t *sp = Wp + blocks * tiles * kMx4PackedTile;
    scale_step = blocks * 256;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int64_t u = u0 + i < 2 * blocks ? u0 + i : 2 * blocks - 1;
      const int64_t b = u >> 1;
      const int row = 16 * (int)(u & 1) + r;
      codes[i] = Wp + b * tiles * kMx4PackedTile + (q >> 1) * 1024 + (q & 1) * 512 + row * 16;
      scales[i] = sp + b * 256 + (q & 1) * 128 + row * 4;
    }
  }
};

// The tokens of MB column blocks: lane column c's row of codes and scales, out
// of range for a column without a token.
template <int MB>
struct Mx4Cols {
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t code_at[MB], scale_at[MB];  // this lane's first bytes, K tile 0
  uint32_t scale_step;
  int blocks;  // blocks of 32 channels in a row

  __device__ __forceinline__ void open(const uint8_t *Xc, const uint8_t *Xe, int64_t rows,
                                       int64_t K) {
    codes = make_rsrc(Xc, (uint32_t)(rows * (K / 2)));
    scales = make_rsrc(Xe, (uint32_t)((K + kMx4Tile - 1) / kMx4Tile * rows * 8));
    scale_step = (uint32_t)rows * 8;
    blocks = (int)(K / 32);
  }
  // column block j's row for this lane (< 0: none)
  __device__ __forceinline__ void aim(int j, int row, int64_t K, int lane) {
    const int q = lane >> 4;
    code_at[j] = row < 0 ? kOobOffset
                         : (uint32_t)row * (uint32_t)(K / 2) + 64 * (q & 1) + 16 * (q >> 1);
    scale_at[j] = row < 0 ? kOobOffset : (uint32_t)row * 8 + 4 * (q & 1);
  }
};

template <int RB, int MB>
struct Mx4Frag {
  v4i a[RB][2], b[MB][2];
  uint32_t ea[RB], eb[MB];
};

template <int RB, int MB>
__device__ __forceinline__ void mx4_load(Mx4Frag<RB, MB> &f, const Mx4Rows<RB> &w,
                                         const Mx4Cols<MB> &x, int t, int lane) {
  const int q = lane >> 4;
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const v4i *p = reinterpret_cast<const v4i *>(w.codes[i] + (int64_t)t * kMx4PackedTile);
    f.a[i][0] = __builtin_nontemporal_load(p);
    f.a[i][1] = __builtin_nontemporal_load(p + 128);
    f.ea[i] = *reinterpret_cast<const uint32_t *>(w.scales[i] + t * w.scale_step);
  }
  const int first = 8 * t + 4 * (q & 1) + (q >> 1);  // this lane's block of instruction 0
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const uint32_t at = x.code_at[j] + (uint32_t)t * kMx4TileBytes;
    f.b[j][0] = __builtin_bit_cast(
        v4i, __builtin_amdgcn_raw_buffer_load_b128(
                 x.codes, x.code_at[j] != kOobOffset && first < x.blocks ? at : kOobOffset, 0, 0));
    f.b[j][1] = __builtin_bit_cast(
        v4i, __builtin_amdgcn_raw_buffer_load_b128(
                 x.codes, x.code_at[j] != kOobOffset && first + 2 < x.blocks ? at + 32 : kOobOffset,
                 0, 0));
    f.eb[j] = __builtin_amdgcn_raw_buffer_load_b32(
        x.scales, x.scale_at[j] != kOobOffset ? x.scale_at[j] + (uint32_t)t * x.scale_step
                                              : kOobOffset, 0, 0);
  }
}

template <int RB, int MB>
__device__ __forceinline__ void mx4_multiply(v4f (&acc)[RB][MB], const Mx4Frag<RB, MB> &f,
                                             int lane) {
  const int down = 8 * (lane >> 5);
  uint32_t ea[RB], eb[MB];
#pragma unroll
  for (int i = 0; i < RB; ++i) ea[i] = f.ea[i] >> down;
#pragma unroll
  for (int j = 0; j < MB; ++j) eb[j] = f.eb[j] >> down;
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j)
      acc[i][j] = mfma_mx4_16<0>(f.a[i][0], f.b[j][0], acc[i][j], ea[i], eb[j]);
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j)
      acc[i][j] = mfma_mx4_16<2>(f.a[i][1], f.b[j][1], acc[i][j], ea[i], eb[j]);
}

// acc += the product over K tiles t0, t0 + step, ... below t1.
template <int RB, int MB, int kDepth>
__device__ __forceinline__ void mx4_stream(v4f (&acc)[RB][MB], const Mx4Rows<RB> &w,
                                           const Mx4Cols<MB> &x, int t0, int t1, int step,
                                           int lane) {
  Mx4Frag<RB, MB> f[kDepth];
#pragma unroll
  for (int d = 0; d < kDepth; ++d)
    if (t0 + d * step < t1) mx4_load(f[d], w, x, t0 + d * step, lane);
  for (int t = t0; t < t1; t += kDepth * step) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (t + d * step < t1) {
        mx4_multiply(acc, f[d], lane);
        if (t + (d + kDepth) * step < t1) mx4_load(f[d], w, x, t + (d + kDepth) * step, lane);
      }
    }
  }
}

}  // namespace detail
}  // namespace ot
