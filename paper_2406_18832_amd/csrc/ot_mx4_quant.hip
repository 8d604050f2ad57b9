// MX4 quantizers: activations, weights (with the activation scale folded in)
// and the way back to values; the packing of weights for the products.
//
// All of it is memory-bound: 2 bytes in and 17/32 of a byte out per element.
// A lane holds eight consecutive channels, a quad of lanes one block: its
// largest magnitude takes two DPP steps on integers (the bits of non-negative
// fp32 values order like the values, and those of a NaN come last), the codes
// four conversions, and each 16 lanes write their four scale bytes as a word.
#include <math.h>

#include "ot_mx4.h"

namespace ot {
namespace detail {

constexpr int kWaves = 4;  // per workgroup, each its own rows

// Runtime activations:  v = fp32(fp32(x - z_k) * inv_s_k), or x itself without
// z and inv_s (SYM false).  As the int8 quantizer: 512 channels to a wave, z and
// inv_s in registers, kRows rows' loads in flight.  MI355X: 4096 x 5120 in 12.7 us
// (4.2 TB/s), 16 x 768 2.4 us, which is a launch.
template <int kRows, bool SYM>
__global__ __launch_bounds__(64 * kWaves) void quantize_act_mx4_kernel(
    const uint16_t *__restrict__ x, int64_t M, int64_t K, const float *__restrict__ z,
    const float *__restrict__ inv_s, uint8_t *__restrict__ Xc, uint8_t *__restrict__ Xe) {
  const int lane = threadIdx.x;
  const int64_t k0 = ((int64_t)blockIdx.x * 64 + lane) * 8;
  const bool in = k0 < K;
  float zr[8], ir[8];
  if constexpr (SYM) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 zz = in ? *reinterpret_cast<const float4 *>(z + k0 + i) : float4{};
      const float4 ii = in ? *reinterpret_cast<const float4 *>(inv_s + k0 + i) : float4{};
      zr[i] = zz.x; zr[i + 1] = zz.y; zr[i + 2] = zz.z; zr[i + 3] = zz.w;
      ir[i] = ii.x; ir[i + 1] = ii.y; ir[i + 2] = ii.z; ir[i + 3] = ii.w;
    }
  }
  const int64_t step = (int64_t)gridDim.y * kWaves;
  for (int64_t g = (int64_t)blockIdx.y * kWaves + threadIdx.y; g * kRows < M; g += step) {
    const int64_t r0 = g * kRows;
    v4u32 w[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      w[u] = in && r0 + u < M
                 ? __builtin_nontemporal_load(reinterpret_cast<const v4u32 *>(x + (r0 + u) * K + k0))
                 : v4u32{0u, 0u, 0u, 0u};
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (r0 + u >= M) break;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = half_bits_to_float((uint16_t)(w[u][i >> 1] >> (16 * (i & 1))));
        if constexpr (SYM) {
          const float t = v[i] - zr[i];  // fp32, RNE
          v[i] = t * ir[i];              // fp32, RNE
        }
      }
      mx4_store8(v, r0 + u, M, K, k0, lane, Xc, Xe);
    }
  }
}

// Offline weights: v = fp32(W[n,k] * s_k), b'_n = fp32(sum_k z_k W[n,k] + b_n)
// with the sum in fp64 (exact products, a fixed order).  kRows rows to a
// workgroup share the reads of s and z, which weigh four times a row of W.
// A row with a non-finite weight, product or bias gets a NaN b' and raises
// *status.
//
// A wave takes 512 channels at a time, all of the row where there are enough
// rows to fill the card with one-wave workgroups (no barrier, and one reduction
// of the fp64 sums to kRows rows), else the waves of a workgroup share the row.
// MI355X: 20480 x 5120 in 66 us (4.0 TB/s; with four waves to four rows 88, with
// four rows to a wave 67, with the next loads ahead of the work 130, for the
// registers), 768 x 768 4.5 us.
constexpr int kFoldWaves = 8;  // at most
constexpr int64_t kFoldGrid = 1 << 20;  // and workgroups; more rows than theirs loop

template <int kRows>
__global__ __launch_bounds__(64 * kFoldWaves, 5) void fold_mx4_kernel(
    const uint16_t *__restrict__ W, const uint16_t *__restrict__ b, int64_t N, int64_t K,
    const float *__restrict__ z, const float *__restrict__ s, uint8_t *__restrict__ Wc,
    uint8_t *__restrict__ We, float *__restrict__ bprime, int *__restrict__ status) {
  __shared__ double red[kFoldWaves][kRows];
  __shared__ int red_bad[kFoldWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, waves = blockDim.x >> 6;
  const int64_t kpad = (K + kMx4Tile - 1) / kMx4Tile * kMx4Tile;
  for (int64_t n0 = (int64_t)blockIdx.x * kRows; n0 < N; n0 += (int64_t)gridDim.x * kRows) {
    double acc[kRows];
    uint32_t bad = 0;  // bit u: row n0 + u
#pragma unroll
    for (int u = 0; u < kRows; ++u) acc[u] = 0.0;
    // whole waves: a lane past the padded end only keeps the others company
    for (int64_t base = (int64_t)wave * 512; base < kpad; base += (int64_t)waves * 512) {
      const int64_t k0 = base + lane * 8;
      const bool in = k0 < K;
      v4u32 w[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u)
        w[u] = in && n0 + u < N
                   ? __builtin_nontemporal_load(reinterpret_cast<const v4u32 *>(W + (n0 + u) * K + k0))
                   : v4u32{0u, 0u, 0u, 0u};
      float sr[8], zr[8];
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 ss = in && s ? *reinterpret_cast<const float4 *>(s + k0 + i)
                                  : make_float4(1.f, 1.f, 1.f, 1.f);
        const float4 zz = in && z ? *reinterpret_cast<const float4 *>(z + k0 + i) : float4{};
        sr[i] = ss.x; sr[i + 1] = ss.y; sr[i + 2] = ss.z; sr[i + 3] = ss.w;
        zr[i] = zz.x; zr[i + 1] = zz.y; zr[i + 2] = zz.z; zr[i + 3] = zz.w;
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (n0 + u >= N) break;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float wk = half_bits_to_float((uint16_t)(w[u][i >> 1] >> (16 * (i & 1))));
          v[i] = wk * sr[i];  // fp32, RNE
          acc[u] = fma((double)zr[i], (double)wk, acc[u]);
        }
        if (mx4_store8(v, n0 + u, N, K, k0, lane, Wc, We) == 255) bad |= 1u << u;
      }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) acc[u] += __shfl_xor(acc[u], off);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) bad |= __shfl_xor(bad, off);
    if (lane == 0) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) red[wave][u] = acc[u];
      red_bad[wave] = (int)bad;
    }
    __syncthreads();
    if (t < kRows && n0 + t < N) {
      double sum = 0.0;
      int any = 0;
      for (int i = 0; i < waves; ++i) {
        sum += red[i][t];
        any |= red_bad[i] >> t & 1;
      }
      const double bn = b ? (double)half_bits_to_float(b[n0 + t]) : 0.0;
      const float r = any ? __builtin_nanf("") : (float)(sum + bn);
      bprime[n0 + t] = r;
      if (status != nullptr && !isfinite(r))
        __hip_atomic_store(status, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    }
    __syncthreads();  // red is free again
  }
}

// Codes to fp32 values: a lane takes four channels, so that the 16-byte stores
// of a wave are one piece of 1 KiB.  MI355X: 20480 x 5120 in 77 us (6.2 TB/s).
constexpr int kDequantRows = 4;

__global__ __launch_bounds__(64 * kWaves) void dequantize_mx4_kernel(
    const uint8_t *__restrict__ c, const uint8_t *__restrict__ e, int64_t rows, int64_t K,
    float *__restrict__ y) {
  const int64_t k0 = ((int64_t)blockIdx.x * 64 + threadIdx.x) * 4;
  if (k0 >= K) return;
  const int64_t step = (int64_t)gridDim.y * kWaves;
  for (int64_t g = (int64_t)blockIdx.y * kWaves + threadIdx.y; g * kDequantRows < rows; g += step) {
    const int64_t r0 = g * kDequantRows;
    uint32_t codes[kDequantRows], b[kDequantRows];
#pragma unroll
    for (int u = 0; u < kDequantRows; ++u) {
      const int64_t row = min(r0 + u, rows - 1);
      codes[u] = *reinterpret_cast<const uint16_t *>(c + row * (K / 2) + k0 / 2);
      b[u] = e[((k0 >> 8) * rows + row) * 8 + ((k0 >> 5) & 7)];
    }
#pragma unroll
    for (int u = 0; u < kDequantRows; ++u) {
      if (r0 + u >= rows) break;
      const float s = mx4_scale(b[u]);
      const v2f lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], s, 0);
      const v2f hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], s, 1);
      float4 v = make_float4(lo[0], lo[1], hi[0], hi[1]);
      if (b[u] == 255) v.x = v.y = v.z = v.w = __builtin_nanf("");
      *reinterpret_cast<float4 *>(y + (r0 + u) * K + k0) = v;
    }
  }
}

// Row-major codes and scales to the packed layout: one 16-byte block of codes
// or one word of scales per thread; a wave reads 16 bytes from each of 32 rows and
// writes 1 KiB.  MI355X: 20480 x 5120 17.8 us (111 MB in and out, in the last-level
// cache: 6.3 TB/s), 9216 x 36864 81 us (361 MB: 4.5 TB/s).
__global__ __launch_bounds__(256) void pack_weights_mx4_kernel(
    const uint8_t *__restrict__ Wc, const uint8_t *__restrict__ We, int64_t N, int64_t K,
    int64_t blocks, int64_t tiles, uint8_t *__restrict__ Wp) {
  const int64_t ncodes = blocks * tiles * 256, nscales = blocks * tiles * 64;
  const int64_t total = ncodes + nscales;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i & 31), h = (int)(i >> 5 & 1);
    if (i < ncodes) {
      const int64_t s = i >> 6 & 3, t = (i >> 8) % tiles, n = (i >> 8) / tiles * 32 + r;
      const int64_t blk = 8 * t + 4 * h + s;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (n < N && blk * 32 < K) v = *reinterpret_cast<const uint4 *>(Wc + n * (K / 2) + blk * 16);
      reinterpret_cast<uint4 *>(Wp)[i] = v;
    } else {
      const int64_t j = i - ncodes;
      const int64_t t = (j >> 6) / blocks, n = (j >> 6) % blocks * 32 + r;
      uint32_t v = 0;
      if (n < N) v = *reinterpret_cast<const uint32_t *>(We + (t * N + n) * 8 + 4 * h);
      reinterpret_cast<uint32_t *>(Wp + ncodes * 16)[j] = v;
    }
  }
}

template <int kRows>
hipError_t launch_qmx4(const uint16_t *x, int64_t M, int64_t K, const float *z, const float *inv_s,
                       uint8_t *Xc, uint8_t *Xe, hipStream_t st) {
  const unsigned gx = (unsigned)((mx4_tiles(K) + 1) / 2);
  int64_t gy = (M + (int64_t)kWaves * kRows - 1) / ((int64_t)kWaves * kRows);
  if (gy > 65535) gy = 65535;
  const dim3 grid(gx, (unsigned)gy), block(64, kWaves);
  if (z)
    quantize_act_mx4_kernel<kRows, true><<<grid, block, 0, st>>>(x, M, K, z, inv_s, Xc, Xe);
  else
    quantize_act_mx4_kernel<kRows, false><<<grid, block, 0, st>>>(x, M, K, z, inv_s, Xc, Xe);
  return hipGetLastError();
}

}  // namespace detail

using namespace detail;

hipError_t launch_quantize_act_mx4(const uint16_t *x, int64_t M, int64_t K, const float *z,
                                   const float *inv_s, uint8_t *Xc, uint8_t *Xe, hipStream_t st) {
  const int64_t row_waves = M * ((mx4_tiles(K) + 1) / 2);
  const int64_t enough = 4 * (int64_t)device_cus();
  if (row_waves >= 8 * enough) return launch_qmx4<8>(x, M, K, z, inv_s, Xc, Xe, st);
  if (row_waves >= 2 * enough) return launch_qmx4<2>(x, M, K, z, inv_s, Xc, Xe, st);
  return launch_qmx4<1>(x, M, K, z, inv_s, Xc, Xe, st);
}

hipError_t launch_fold_mx4(const uint16_t *W, const uint16_t *b, int64_t N, int64_t K,
                           const float *z, const float *s, uint8_t *Wc, uint8_t *We,
                           float *bprime, int *status, hipStream_t st) {
  constexpr int kRows = 2;
  int64_t grid = (N + kRows - 1) / kRows;
  const int64_t pieces = (mx4_tiles(K) + 1) / 2, wanted = 20 * (int64_t)device_cus();
  int64_t waves = (wanted + grid - 1) / grid;
  if (waves > kFoldWaves) waves = kFoldWaves;
  const int64_t rounds = (pieces + waves - 1) / waves;
  waves = (pieces + rounds - 1) / rounds;
  if (grid > kFoldGrid) grid = kFoldGrid;
  fold_mx4_kernel<kRows><<<(unsigned)grid, (unsigned)(64 * waves), 0, st>>>(
      W, b, N, K, z, s, Wc, We, bprime, status);
  return hipGetLastError();
}

hipError_t launch_dequantize_mx4(const uint8_t *c, const uint8_t *e, int64_t rows, int64_t K,
                                 float *y, hipStream_t st) {
  const unsigned gx = (unsigned)((K / 4 + 63) / 64);
  int64_t gy = (rows + kWaves * kDequantRows - 1) / (kWaves * kDequantRows);
  if (gy > 65535) gy = 65535;
  dequantize_mx4_kernel<<<dim3(gx, (unsigned)gy), dim3(64, kWaves), 0, st>>>(c, e, rows, K, y);
  return hipGetLastError();
}

hipError_t launch_pack_weights_mx4(const uint8_t *Wc, const uint8_t *We, int64_t N, int64_t K,
                                   uint8_t *Wp, hipStream_t st) {
  const int64_t blocks = (N + 31) / 32, tiles = mx4_tiles(K);
  int64_t grid = (blocks * tiles * 320 + 255) / 256;
  if (grid > (int64_t)device_cus() * 64) grid = (int64_t)device_cus() * 64;
  pack_weights_mx4_kernel<<<(unsigned)grid, 256, 0, st>>>(Wc, We, N, K, blocks, tiles, Wp);
  return hipGetLastError();
}

}  // namespace ot
