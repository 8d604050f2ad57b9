// MX4: the microscaled 4-bit floating point format of the mx4 entry points,
// and the device helpers that their kernels share.
//
// A block of 32 consecutive channels holds one e8m0 scale byte b, worth
// 2^(b-127) (255: the whole block is NaN), and 32 e2m1 codes: a sign and one
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  With E the exponent field of the largest
// fp32 magnitude in the block,
//   b = max(E - 2, 0), 255 where E = 255 (an infinity or a NaN in the block)
//   code = the level nearest to v 2^(127-b), ties to the even code, at most 6
// so that the largest magnitude lands in [4, 8) before rounding (values past 6
// saturate, as the format's own rule has it).  v_cvt_scalef32_pk_fp4_f32 is
// that division, rounding and saturation, down to b = 0 (checked on gfx950 for
// every level, tie and neighbour of a tie).
//
// Layouts.  Codes [rows][K/2] bytes, the even channel in the low half; scales
// [ceil(K/256)][rows][8] bytes (a K tile's eight scales of a row side by side,
// zeros past K), so that a K tile of a GEMM's rows is one contiguous piece.
// Packed weights: mx4_packed_bytes() below.
#pragma once

#include "ot_gemm_common.h"

namespace ot {

constexpr int kMx4Tile = 256;        // channels per K tile
constexpr int kMx4TileBytes = 128;   // their codes in a row
constexpr int kMx4PackedTile = 4096; // codes of a packed 32-row K tile
constexpr int64_t kMx4MaxK = int64_t(1) << 22;

inline int64_t mx4_tiles(int64_t K) { return (K + kMx4Tile - 1) / kMx4Tile; }

// Packed weights: with T = ceil(K/256), B = ceil(N/32), first the codes
//   [B][T][4 steps s][2 halves h][32 rows r][16 bytes], block 8t + 4h + s of row
// (1 KiB per step: one wave's operand of v_mfma_scale_f32_32x32x64_f8f6f4, whose
// lane 32h + r holds 32 channels of row r), then the scales
//   [T][B][2 halves][32 rows][4 steps]
// (a lane's scales of a tile's four steps in one word), zeros past N and K.
inline size_t mx4_packed_bytes(int64_t N, int64_t K) {
  return (size_t)((N + 31) / 32) * (size_t)mx4_tiles(K) * (kMx4PackedTile + 256);
}

namespace detail {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u32 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale byte of a block whose largest magnitude has these bits.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t most) {
  const int e = (int)(most >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
// 2^(b-127) for b < 255 (b = 0: the subnormal 2^-127).
__device__ __forceinline__ float mx4_scale(uint32_t b) {
  return __uint_as_float(b ? b << 23 : 0x00400000u);
}

// The codes of eight values, value i in bits 4i .. 4i+3.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t b) {
  const float s = mx4_scale(b);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return b == 255 ? 0u : c;
}

// Maximum over, and OR along, the 4 lanes of a quad / the 16 of a row (DPP: no
// LDS).  All 64 lanes take part.
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp<0xB1>(v));  // quad_perm 1, 0, 3, 2
  return max(v, dpp<0x4E>(v));  // quad_perm 2, 3, 0, 1
}
// The scale bytes of a row's four quads (blocks) as one word, in every lane.
__device__ __forceinline__ uint32_t row_scales(uint32_t b, int lane) {
  uint32_t w = b << (8 * ((lane >> 2) & 3));
  w |= dpp<0x124>(w);  // row_ror:4
  return w | dpp<0x128>(w);  // row_ror:8
}

// Lane l of a wave holds eight consecutive channels from k0 = 8 (64 i + l) on,
// zeros past K: their codes and scales to row `row` of [M x K].  All 64 lanes
// take part.  The scale byte of the lane's block.
__device__ __forceinline__ uint32_t mx4_store8(const float (&v)[8], int64_t row, int64_t M,
                                               int64_t K, int64_t k0, int lane,
                                               uint8_t *__restrict__ Xc, uint8_t *__restrict__ Xe) {
  uint32_t most = abs_bits(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) most = max(most, abs_bits(v[i]));
  const uint32_t b = mx4_scale_byte(quad_max(most));
  const uint32_t e = row_scales(b, lane);
  if (k0 < K) *reinterpret_cast<uint32_t *>(Xc + row * (K / 2) + k0 / 2) = mx4_codes8(v, b);
  // one lane of 16 (128 channels) writes their four scales, also past K up to
  // the end of the K tile
  if ((lane & 15) == 0 && k0 < (K + kMx4Tile - 1) / kMx4Tile * kMx4Tile)
    *reinterpret_cast<uint32_t *>(Xe + ((k0 >> 8) * M + row) * 8 + ((k0 >> 5) & 7)) = e;
  return b;
}

}  // namespace detail

hipError_t launch_quantize_act_mx4(const uint16_t *x, int64_t M, int64_t K, const float *z,
                                   const float *inv_s, uint8_t *Xc, uint8_t *Xe, hipStream_t st);
hipError_t launch_ln_quantize_act_mx4(const uint16_t *h, int64_t M, int64_t K,
                                      const uint16_t *gamma, const uint16_t *beta, float eps,
                                      const float *z, const float *inv_s, uint8_t *Xc, uint8_t *Xe,
                                      hipStream_t st);
// status as for launch_fold; z and s: either may be NULL.
hipError_t launch_fold_mx4(const uint16_t *W, const uint16_t *b, int64_t N, int64_t K,
                           const float *z, const float *s, uint8_t *Wc, uint8_t *We,
                           float *bprime, int *status, hipStream_t st);
hipError_t launch_dequantize_mx4(const uint8_t *c, const uint8_t *e, int64_t rows, int64_t K,
                                 float *y, hipStream_t st);
hipError_t launch_pack_weights_mx4(const uint8_t *Wc, const uint8_t *We, int64_t N, int64_t K,
                                   uint8_t *Wp, hipStream_t st);

// Estimated time of a launch in microseconds: passes over the CUs, each of `pass`
// and `per_k` per K tile, plus `share` per K tile for the workgroups' mean number
// per CU (what they take from each other), plus `once`.
struct Mx4Time {
  double once, pass, per_k, share;
  double us(int64_t workgroups, int64_t k_tiles, int64_t cus) const {
    const double passes = (double)((workgroups + cus - 1) / cus), kt = (double)k_tiles;
    return once + passes * (pass + per_k * kt) + share * kt * (double)workgroups / (double)cus;
  }
};

// A launch of the tile kernels: its tile, the parts that K is shared out to, the
// workspace for their sums and the estimated time.
struct Mx4Plan {
  int tile, bn, bm, parts;
  size_t bytes;
  double us;
};
Mx4Plan mx4_gemm_plan(int64_t M, int64_t N, int64_t K, bool with_workspace);
hipError_t launch_mx4_gemm(const Mx4Plan &plan, const uint8_t *Xc, const uint8_t *Xe,
                           const uint8_t *Wp, const float *bp, int64_t M, int64_t N, int64_t K,
                           uint16_t *Y, void *ws, hipStream_t st);
bool mx4_gemm_fits(int64_t M, int64_t N);  // whether some tile's grid does
// Whether a launch of these sizes, or of more tokens, can share K at all.
bool mx4_gemm_may_share(int64_t M, int64_t N, int64_t K);

// The product: up to 64 tokens mostly by streaming the weights
// (ot_mx4_decode.hip), else on tiles.  ws: NULL or mx4_linear_workspace_bytes.
hipError_t launch_mx4_linear(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                             const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                             void *ws, hipStream_t st);
size_t mx4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);
size_t mx4_linear_workspace_max(int64_t M, int64_t N, int64_t K);
void describe_mx4_linear(int64_t M, int64_t N, int64_t K, bool with_workspace, char *buf,
                         size_t len);
// A mixture-of-experts layer; workspace of at least moe_mx4_workspace_bytes.
size_t moe_mx4_workspace_bytes(int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k);
hipError_t launch_moe_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint16_t *logits,
                          const uint8_t *W1, const float *b1, const uint8_t *W2, const float *b2,
                          int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k, bool glu,
                          uint16_t *Y, void *workspace, hipStream_t st);

}  // namespace ot
