// The MX4 linear up to 64 tokens:  Y = fp16(sum_k x w + b').
//
// Bound by reading the weights (MI355X: 8 tokens x 20480, K = 5120 in 11.5 us, 4.9
// TB/s; 14336 x 28928 with 3 tokens 34 us, 6.4).  A workgroup takes 16 RB weight rows and all
// tokens; its waves share out the K tiles and add their fp32 sums through LDS
// in wave order (ot_mx4_stream.h).
//
// Up to 16 tokens a wave loads the tokens' codes straight into registers.  With
// more, those loads (pieces of 32 bytes from each of 16 rows) cost more than the
// weights': there the wave copies its K tile of all tokens into LDS of its own,
// whole 128-byte row pieces at a time, and takes the fragments from there.  No
// wave waits for another before the sums meet.
#include <stdio.h>

#include "ot_mx4_stream.h"
#include "ot_mx4_tiles.h"

namespace ot {
namespace detail {

// Adds the waves' sums, in wave order, and writes the outputs.  red: [waves][RB]
// [MB][64]; lane l of block (i, j) holds token 16 j + l mod 16 and rows
// 4 (l / 16) .. +3 of unit u0 + i.
template <int RB, int MB>
__device__ __forceinline__ void mx4_decode_finish(const v4f (&acc)[RB][MB], v4f *red, int64_t u0,
                                                  const float *__restrict__ bp, int M, int N,
                                                  uint16_t *__restrict__ Y, int wave, int waves,
                                                  int lane) {
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) red[((wave * RB + i) * MB + j) * 64 + lane] = acc[i][j];
  __syncthreads();
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

// Up to 16 tokens.
template <int RB, int kMaxWaves>
__global__ __launch_bounds__(64 * kMaxWaves) void mx4_decode_kernel(
    const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe, const uint8_t *__restrict__ Wp,
    const float *__restrict__ bp, int M, int N, int K, int tiles, uint16_t *__restrict__ Y) {
  extern __shared__ v4f red[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int64_t u0 = (int64_t)blockIdx.x * RB;
  Mx4Rows<RB> w;
  w.aim(Wp, (N + 31) / 32, tiles, u0, lane);
  Mx4Cols<1> x;
  x.open(Xc, Xe, M, K);
  x.aim(0, (lane & 15) < M ? lane & 15 : -1, K, lane);
  v4f acc[RB][1];
#pragma unroll
  for (int i = 0; i < RB; ++i) acc[i][0] = v4f{0.f, 0.f, 0.f, 0.f};
  mx4_stream<RB, 1, 2>(acc, w, x, wave, tiles, waves, lane);
  mx4_decode_finish<RB, 1>(acc, red, u0, bp, M, N, Y, wave, waves, lane);
}

// 17 to 16 MB tokens: a wave's LDS is its K tile of 16 MB token rows, 128 bytes
// each, 16-byte chunk c of row r at chunk c ^ swz_mx4(r).
template <int RB, int MB>
struct Mx4LdsFrag {
  v4i a[RB][2];
  uint32_t ea[RB], eb[MB];
};

template <int RB, int MB, int kMaxWaves>
__global__ __launch_bounds__(64 * kMaxWaves) void mx4_decode_lds_kernel(
    const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe, const uint8_t *__restrict__ Wp,
    const float *__restrict__ bp, int M, int N, int K, int tiles, uint16_t *__restrict__ Y) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int64_t u0 = (int64_t)blockIdx.x * RB;
  const int r = lane & 15, q = lane >> 4, KB = K / 2;
  Mx4Rows<RB> w;
  w.aim(Wp, (N + 31) / 32, tiles, u0, lane);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(Xc, (uint32_t)(M * KB));
  const __amdgpu_buffer_rsrc_t re = make_rsrc(Xe, (uint32_t)(tiles * M * 8));
  uint8_t *const own = lds + wave * (MB * 2048);
  // rows 8 j + lane / 8: the swizzle of their chunk goes by 8 (j mod 2)
  const int row8 = lane >> 3;
  const int ck0 = ((lane & 7) ^ swz_mx4(row8)) * 16, ck1 = ((lane & 7) ^ swz_mx4(8 + row8)) * 16;
  int off_f[2];
#pragma unroll
  for (int p = 0; p < 2; ++p)
    off_f[p] = r * 128 + 16 * ((4 * (q & 1) + 2 * p + (q >> 1)) ^ swz_mx4(r));

  // K tile t: the tokens to LDS, then the weights and scales to registers
  auto issue = [&](Mx4LdsFrag<RB, MB> &f, int t) {
    const int k0 = t * kMx4TileBytes;
#pragma unroll
    for (int j = 0; j < 2 * MB; ++j) {
      const int ck = j & 1 ? ck1 : ck0;
      if (8 * j < M)  // the other rows' columns are never written
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rx, (lds_void *)(own + j * 1024), 16,
            k0 + ck < KB ? (uint32_t)((8 * j + row8) * KB + k0 + ck) : kOobOffset, 0, 0, 0);
    }
    asm volatile("" ::: "memory");  // the copies are the older loads
#pragma unroll
    for (int j = 0; j < MB; ++j)
      f.eb[j] = __builtin_amdgcn_raw_buffer_load_b32(
          re, (uint32_t)(t * M + 16 * j + r) * 8 + 4 * (q & 1), 0, 0);
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const v4i *p = reinterpret_cast<const v4i *>(w.codes[i] + (int64_t)t * kMx4PackedTile);
      f.ea[i] = *reinterpret_cast<const uint32_t *>(w.scales[i] + t * w.scale_step);
      f.a[i][0] = __builtin_nontemporal_load(p);
      f.a[i][1] = __builtin_nontemporal_load(p + 128);
    }
    asm volatile("" ::: "memory");
  };
  v4f acc[RB][MB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  // The tile in f: once its weights are here (loads return in order) the older
  // copies have landed.  The tokens' fragments out of LDS, then the next tile's
  // loads, then the products.
  auto step = [&](Mx4LdsFrag<RB, MB> &f, Mx4LdsFrag<RB, MB> &next, int t) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
      asm volatile("" : "+v"(f.a[i][0]), "+v"(f.a[i][1]), "+v"(f.ea[i])::"memory");
    v4i b[MB][2];
#pragma unroll
    for (int j = 0; j < MB; ++j)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        b[j][p] = *reinterpret_cast<const v4i *>(own + j * 2048 + off_f[p]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // before the copies below
#pragma unroll
    for (int j = 0; j < MB; ++j) asm volatile("" : "+v"(b[j][0]), "+v"(b[j][1])::"memory");
    if (t + waves < tiles) issue(next, t + waves);
    const int down = 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < MB; ++j)
        acc[i][j] = mfma_mx4_16<0>(f.a[i][0], b[j][0], acc[i][j], f.ea[i] >> down, f.eb[j] >> down);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < MB; ++j)
        acc[i][j] = mfma_mx4_16<2>(f.a[i][1], b[j][1], acc[i][j], f.ea[i] >> down, f.eb[j] >> down);
  };
  Mx4LdsFrag<RB, MB> f0, f1;
  if (wave < tiles) issue(f0, wave);
  for (int t = wave; t < tiles; t += 2 * waves) {
    step(f0, f1, t);
    if (t + waves < tiles) step(f1, f0, t + waves);
  }
  __syncthreads();  // the waves' LDS becomes the sums'
  mx4_decode_finish<RB, MB>(acc, reinterpret_cast<v4f *>(lds), u0, bp, M, N, Y, wave, waves, lane);
}

// Waves of a workgroup: as many as share the K tiles evenly.
template <int kMaxWaves>
int decode_waves(int tiles) {
  const int rounds = (tiles + kMaxWaves - 1) / kMaxWaves;
  return (tiles + rounds - 1) / rounds;
}

template <int RB, int kMaxWaves>
hipError_t launch_decode(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp, const float *bp,
                         int64_t M, int64_t N, int64_t K, uint16_t *Y, hipStream_t st) {
  const int tiles = (int)mx4_tiles(K), waves = decode_waves<kMaxWaves>(tiles);
  const unsigned grid = (unsigned)(((N + 15) / 16 + RB - 1) / RB);
  mx4_decode_kernel<RB, kMaxWaves><<<grid, 64 * waves, (size_t)waves * RB * 1024, st>>>(
      Xc, Xe, Wp, bp, (int)M, (int)N, (int)K, tiles, Y);
  return hipGetLastError();
}

template <int RB, int MB, int kMaxWaves>
hipError_t launch_decode_lds(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                             const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                             hipStream_t st) {
  static_assert(RB <= 2, "the sums fit the waves' LDS");
  const int tiles = (int)mx4_tiles(K), waves = decode_waves<kMaxWaves>(tiles);
  const unsigned grid = (unsigned)(((N + 15) / 16 + RB - 1) / RB);
  mx4_decode_lds_kernel<RB, MB, kMaxWaves><<<grid, 64 * waves, (size_t)waves * MB * 2048, st>>>(
      Xc, Xe, Wp, bp, (int)M, (int)N, (int)K, tiles, Y);
  return hipGetLastError();
}

}  // namespace detail

using namespace detail;

// Which kernel.  Up to 16 tokens 16 rows to a workgroup where that is at most one
// of them per CU (more, and they read the tokens too often), or where the whole
// launch is latency; else 32.  On MI355X, 16 and 32 rows: 9 x 3466, K = 24416 12.0
// and 15.6 us; 16 x 5120, K = 20480 20.2 and 15.2; 8 x 20480, K = 5120 14.0 and
// 12.2; 2 x 4352, K = 1024 3.0 and 3.2; over 50 random launches 0.6 % over the
// faster one.
// From 17 on whichever of these and the tiles of ot_mx4_gemm.hip (which read the
// tokens once per 64 or 128 rows) is estimated to be the fastest.  Fitted to 110
// random launches, where the choice is 0.9 % over the fastest (15 % at worst); 32 x
// 5120, K = 20480: 16 rows 21, 32 rows 16.1, tiles 25.2 or, in 3 parts, 16.7; 64 x
// 20480, K = 5120: 23.8, 21.7 and 15.2; 54 x 4736, K = 1248: 4.3, 4.4 and 4.8.
static constexpr Mx4Time kDecodeTime[2][2] = {  // [17 .. 32, 33 .. 64][16, 32 rows]
    {{2.779, 0.041, 0.112, 0.004}, {2.959, 0.221, 0.134, 0.045}},
    {{2.418, 0.304, 0.140, 0.043}, {2.523, 1.034, 0.150, 0.119}},
};

// rows: of a workgroup, or 0 for the tiles.
struct LinearPlan {
  int rows;
  Mx4Plan tiles;
};
static LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, bool with_workspace) {
  const int64_t cus = device_cus();
  if (M <= 16)
    return {N <= 16 * cus || N * K < (int64_t(1) << 24) ? 16 : 32, Mx4Plan{}};
  LinearPlan plan{0, mx4_gemm_plan(M, N, K, with_workspace)};
  if (M > 64) return plan;
  double least = plan.tiles.us;
  for (int i = 0; i < 2; ++i) {
    const int rows = 16 << i;
    const double us = kDecodeTime[M > 32][i].us((N + rows - 1) / rows, mx4_tiles(K), cus);
    if (us < least) {
      plan.rows = rows;
      least = us;
    }
  }
  return plan;
}

size_t mx4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  const LinearPlan plan = linear_plan(M, N, K, true);
  return plan.rows ? 0 : plan.tiles.bytes;
}

// The most that any call of 1 to M tokens uses: a plan is the same for all tokens
// of one count of 64-row tiles, and for 17 to 32.
size_t mx4_linear_workspace_max(int64_t M, int64_t N, int64_t K) {
  size_t most = 0;
  for (int64_t m = 32; mx4_gemm_may_share(m < M ? m : M, N, K); m += m < 64 ? 32 : 64) {
    const size_t bytes = mx4_linear_workspace_bytes(m < M ? m : M, N, K);
    if (bytes > most) most = bytes;
    if (m >= M) break;
  }
  return most;
}

void describe_mx4_linear(int64_t M, int64_t N, int64_t K, bool with_workspace, char *buf,
                         size_t len) {
  const LinearPlan plan = linear_plan(M, N, K, with_workspace);
  if (plan.rows)
    snprintf(buf, len, "decode %d rows", plan.rows);
  else if (plan.tiles.parts > 1)
    snprintf(buf, len, "tiles %dx%d split-K %d", plan.tiles.bn, plan.tiles.bm, plan.tiles.parts);
  else
    snprintf(buf, len, "tiles %dx%d", plan.tiles.bn, plan.tiles.bm);
}

hipError_t launch_mx4_linear(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                             const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                             void *ws, hipStream_t st) {
  const LinearPlan plan = linear_plan(M, N, K, ws != nullptr);
  if (plan.rows == 0) return launch_mx4_gemm(plan.tiles, Xc, Xe, Wp, bp, M, N, K, Y, ws, st);
  const bool narrow = plan.rows == 16;
  if (M <= 16)
    return narrow ? launch_decode<1, 16>(Xc, Xe, Wp, bp, M, N, K, Y, st)
                  : launch_decode<2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
  if (M <= 32)
    return narrow ? launch_decode_lds<1, 2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st)
                  : launch_decode_lds<2, 2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
  return narrow ? launch_decode_lds<1, 4, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st)
                : launch_decode_lds<2, 4, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
}

}  // namespace ot
