// The MX4 linear up to 64 tokens:  Y = fp16(sum_k x w + b').
//
// Bound by reading the weights.  A workgroup takes 16 RB weight rows and all
// tokens; its waves share out the K tiles and add their fp32 sums through LDS
// in wave order (ot_mx4_stream.h).
#include "ot_mx4_stream.h"

namespace ot {
namespace detail {

template <int RB, int MB, int kDepth, int kMaxWaves>
__global__ __launch_bounds__(64 * kMaxWaves) void mx4_decode_kernel(
    const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe, const uint8_t *__restrict__ Wp,
    const float *__restrict__ bp, int M, int N, int K, int tiles, uint16_t *__restrict__ Y) {
  extern __shared__ v4f red[];  // [waves][RB][MB][64]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int64_t u0 = (int64_t)blockIdx.x * RB;

  Mx4Rows<RB> w;
  w.aim(Wp, (N + 31) / 32, tiles, u0, lane);
  Mx4Cols<MB> x;
  x.open(Xc, Xe, M, K);
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const int m = 16 * j + (lane & 15);
    x.aim(j, m < M ? m : -1, K, lane);
  }
  v4f acc[RB][MB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  mx4_stream<RB, MB, kDepth>(acc, w, x, wave, tiles, waves, lane);
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) red[((wave * RB + i) * MB + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  // item o: lane l of block (i, j) holds token 16 j + l mod 16 and rows
  // 4 (l / 16) .. +3 of unit i
  for (int o = threadIdx.x; o < RB * MB * 64; o += blockDim.x) {
    v4f s = red[o];
    for (int v = 1; v < waves; ++v) s += red[v * RB * MB * 64 + o];
    const int l = o & 63, j = (o >> 6) % MB, i = (o >> 6) / MB;
    const int64_t m = 16 * j + (l & 15), n = (u0 + i) * 16 + 4 * (l >> 4);
    if (m >= M || n >= N) continue;
    uint16_t *dst = Y + m * N + n;
    if (n + 3 < N && (N & 3) == 0) {
      const float4 b4 = *reinterpret_cast<const float4 *>(bp + n);
      uint2 h;
      h.x = (uint32_t)float_to_half_bits(s[0] + b4.x) |
            ((uint32_t)float_to_half_bits(s[1] + b4.y) << 16);
      h.y = (uint32_t)float_to_half_bits(s[2] + b4.z) |
            ((uint32_t)float_to_half_bits(s[3] + b4.w) << 16);
      *reinterpret_cast<uint2 *>(dst) = h;
    } else {
      for (int e = 0; e < 4; ++e)
        if (n + e < N) dst[e] = float_to_half_bits(s[e] + bp[n + e]);
    }
  }
}

template <int RB, int MB, int kDepth, int kMaxWaves>
hipError_t launch_decode(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp, const float *bp,
                         int64_t M, int64_t N, int64_t K, uint16_t *Y, hipStream_t st) {
  const int tiles = (int)mx4_tiles(K);
  // waves: as many as share the K tiles evenly
  const int rounds = (tiles + kMaxWaves - 1) / kMaxWaves;
  const int waves = (tiles + rounds - 1) / rounds;
  const unsigned grid = (unsigned)(((N + 15) / 16 + RB - 1) / RB);
  mx4_decode_kernel<RB, MB, kDepth, kMaxWaves>
      <<<grid, 64 * waves, (size_t)waves * RB * MB * 1024, st>>>(Xc, Xe, Wp, bp, (int)M, (int)N,
                                                                 (int)K, tiles, Y);
  return hipGetLastError();
}

}  // namespace detail

using namespace detail;

hipError_t launch_mx4_decode(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                             const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                             hipStream_t st) {
  if (M <= 16) return launch_decode<1, 1, 4, 16>(Xc, Xe, Wp, bp, M, N, K, Y, st);
  if (M <= 32) return launch_decode<2, 2, 2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
  return launch_decode<2, 4, 2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
}

}  // namespace ot
