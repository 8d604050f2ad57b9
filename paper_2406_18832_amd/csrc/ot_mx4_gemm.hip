// The MX4 linear above 64 tokens, and below where it is the faster:
//   Y = fp16(sum_k x w + b')
// with both operands in MX4 (ot_mx4.h), products and scales on
// v_mfma_scale_f32_32x32x64_f8f6f4, sums in fp32.
//
// The matrix instruction takes 16 bytes of codes per lane (a block of 32
// channels) and one scale byte per lane and operand, and does twice the work of
// the int8 one in the same cycles, so the tile walk, LDS staging and epilogue
// are those of the int8 prefill with a byte of codes standing for two channels:
// workgroup tile BN (weight rows) x BM (token rows), K tiles of 256 channels (128
// bytes of a row), S of them in a ring, filled by buffer loads straight to LDS.
//
// A K tile's blocks go to the matrix steps so that step s takes blocks s and
// 4 + s (lane half h takes 4h + s): a lane's four scales of a tile are then one
// 32-bit word, from which each step picks its byte by an immediate.
//   weights  packed in operand order: a step of 32 rows is 1 KiB, copied and
//            read without a swizzle
//   tokens   row-major: 16-byte chunk c of row r at chunk c ^ swz(r)
//   scales   a word per lane and 32 rows, read once per K tile
//
// MI355X: 9216 x 36864 with 8192 tokens in 1230-1270 us, 4.4-4.5 PFLOP/s: the matrix
// cores are busy 64 % of the time at the 1.67 GHz that power leaves; a loop of these
// instructions on random registers alone reaches 6.6.
#include "ot_mx4_tiles.h"

namespace ot {
namespace detail {

template <int BN, int BM, int WN, int WM, int S>
struct Mx4Cfg {
  static constexpr int kWaves = WN * WM;
  static constexpr int kTN = BN / WN, kTM = BM / WM;
  static constexpr int kFN = kTN / 32, kFM = kTM / 32;
  static constexpr int kABytes = BN * 128, kBBytes = BM * 128;
  static constexpr int kScaleA = kABytes + kBBytes, kScaleB = kScaleA + BN * 8;
  static constexpr int kStage = kScaleB + BM * 8;
  static constexpr int kLoadsA = BN / 8 / kWaves, kLoadsB = BM / 8 / kWaves;  // 1 KiB each
  static constexpr int kPieces = (BN + BM) / 32;  // of scales, 256 bytes (32 rows) each
  static constexpr int kLoadsE = (kPieces + kWaves - 1) / kWaves;
  static constexpr int kLoads = kLoadsA + kLoadsB + kLoadsE;
  static constexpr int kMfma = kFN * kFM, kReads = kFN + kFM;
  static constexpr int kOut = BN * BM * 2;  // the fp16 output tile, staged after the loop
  static constexpr int kSmem = S * kStage > kOut ? S * kStage : kOut;
  static_assert(kLoadsA * 8 * kWaves == BN && kLoadsB * 8 * kWaves == BM, "whole code loads");
  static_assert(kTN % 32 == 0 && kTM % 32 == 0, "32x32 blocks");
  static_assert(S >= 2 && (S - 2) * kLoads <= 63, "vmcnt range");
  static_assert(kSmem <= 160 * 1024, "LDS");
};

// PARTS false: all of K, to Y.  PARTS true: workgroups of `parts` equal shares of
// the K tiles, whose fp32 sums go to `sums` as mx4_join_kernel reads them.
template <int BN, int BM, int WN, int WM, int S, bool PARTS>
__device__ __forceinline__ void mx4_gemm_body(
    uint8_t *smem, const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe,
    const uint8_t *__restrict__ Wp, const float *__restrict__ bp, int M, int N, int K,
    uint16_t *__restrict__ Y, int tiles_m, int tiles_n, int parts, v4f *__restrict__ sums) {
  using C = Mx4Cfg<BN, BM, WN, WM, S>;
  const int KB = K / 2;                      // bytes of a token row
  const int KT = (K + kMx4Tile - 1) / kMx4Tile;
  const int NB = (N + 31) / 32;              // 32-row blocks of the packed weights

  const TilePlace place(tiles_m, tiles_n, PARTS);
  const int tm = place.tm, tn = place.tn;
  const int kt0 = PARTS ? place.part * KT / parts : 0;               // its K tiles
  const int kn = PARTS ? (place.part + 1) * KT / parts - kt0 : KT;
  const int n0 = tn * BN, m0 = tm * BM;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wm = wave / WN;

  // ---- global -> LDS --------------------------------------------------------
  const int blocks_a = min(BN / 32, NB - tn * (BN / 32));
  const int rows_b = min(BM, M - m0);
  const uint8_t *scales_w = Wp + (int64_t)NB * KT * kMx4PackedTile + (int64_t)(n0 / 32) * 256;
  const uint8_t *scales_x = Xe + (int64_t)m0 * 8;
  const __amdgpu_buffer_rsrc_t rsrc_a =
      make_rsrc(Wp + (int64_t)(n0 / 32) * KT * kMx4PackedTile,
                (uint32_t)blocks_a * (uint32_t)KT * kMx4PackedTile);
  const __amdgpu_buffer_rsrc_t rsrc_b =
      make_rsrc(Xc + (int64_t)m0 * KB, (uint32_t)rows_b * (uint32_t)KB);
  // weights: 1 KiB load q is step q mod 4 of block q / 4
  uint32_t off_a[C::kLoadsA], off_b[C::kLoadsB];
#pragma unroll
  for (int j = 0; j < C::kLoadsA; ++j) {
    const int q = wave * C::kLoadsA + j;
    off_a[j] = (uint32_t)(q >> 2) * (uint32_t)KT * kMx4PackedTile + (q & 3) * 1024 + lane * 16;
  }
  // tokens: a 1 KiB load is 8 rows of 8 chunks; the rows of a lane's loads are a
  // multiple of 8 apart, so two chunk positions serve them all
  int ck_b[C::kLoadsB];
#pragma unroll
  for (int j = 0; j < C::kLoadsB; ++j) {
    const int row = (wave * C::kLoadsB + j) * 8 + lane / 8;
    ck_b[j] = ((lane & 7) ^ swz_mx4(row)) * 16;
    off_b[j] = (uint32_t)row * (uint32_t)KB + ck_b[j];
  }
  // Load j of its K tile kt into its stage.  Tiles past the end load zeros (out
  // of range) into stages that nobody reads, so that every iteration has the
  // same number of loads in flight.
  auto issue_one = [&](int kt, int j) {
    uint8_t *st = smem + (kt % S) * C::kStage;
    if (j < C::kLoadsA) {
      const int ja = j < C::kLoadsA ? j : 0;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc_a, (lds_void *)(st + (wave * C::kLoadsA + ja) * 1024), 16,
          kt < kn ? off_a[ja] + (uint32_t)(kt0 + kt) * kMx4PackedTile : kOobOffset, 0, 0, 0);
    } else if (j < C::kLoadsA + C::kLoadsB) {
      const int jb = j >= C::kLoadsA && j < C::kLoadsA + C::kLoadsB ? j - C::kLoadsA : 0;
      const int k0 = (kt0 + kt) * kMx4TileBytes;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc_b, (lds_void *)(st + C::kABytes + (wave * C::kLoadsB + jb) * 1024), 16,
          kt < kn && k0 + ck_b[jb] < KB ? off_b[jb] + (uint32_t)k0 : kOobOffset, 0, 0, 0);
    } else {
      // Scales: 256-byte piece q, of 32 weight rows or 32 token rows (waves left
      // over load the last one once more).  By 4 bytes a lane, since an odd number
      // of token rows leaves no wider alignment.  Fewer waves copying a KiB each
      // saved loads and cost more (OPT-66B fc2, 8192 tokens: 1229 us, and 1260 so).
      const int q = min(wave * C::kLoadsE + (j - C::kLoadsA - C::kLoadsB), C::kPieces - 1);
      const int t = kt0 + min(kt, kn - 1);
      if (q < BN / 32) {
        const __amdgpu_buffer_rsrc_t r =
            make_rsrc(scales_w + (int64_t)t * NB * 256, (uint32_t)blocks_a * 256);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(st + C::kScaleA + q * 256), 4,
                                                 q * 256 + lane * 4, 0, 0, 0);
      } else {
        const int qb = q - BN / 32;
        const __amdgpu_buffer_rsrc_t r =
            make_rsrc(scales_x + (int64_t)t * M * 8, (uint32_t)rows_b * 8);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(st + C::kScaleB + qb * 256), 4,
                                                 qb * 256 + lane * 4, 0, 0, 0);
      }
    }
  };

  // ---- LDS -> registers -----------------------------------------------------
  const int fr = lane & 31, fh = lane >> 5;
  int off_f[4];  // token fragment: row fr, chunk 4h + s
#pragma unroll
  for (int s = 0; s < 4; ++s) off_f[s] = fr * 128 + 16 * ((4 * fh + s) ^ swz_mx4(fr));
  const int a_base = wn * C::kFN * kMx4PackedTile + lane * 16;
  const int b_base = C::kABytes + wm * C::kTM * 128;
  const int ea_base = C::kScaleA + wn * C::kTN * 8 + lane * 4;
  const int eb_base = C::kScaleB + wm * C::kTM * 8 + fr * 8 + fh * 4;

  v4i fa[2][C::kFN], fb[2][C::kFM];
  int ea[C::kFN], eb[C::kFM], na[C::kFN], nb[C::kFM];
  v16f acc[C::kFN][C::kFM];
#pragma unroll
  for (int f = 0; f < C::kFN; ++f)
#pragma unroll
    for (int g = 0; g < C::kFM; ++g) acc[f][g] = v16f{};

  // A K tile's loads are spread evenly over the MFMAs from the previous tile's
  // last step to its own last but one; upto(u) of them go out before the u-th.
  constexpr int kSlots = C::kMfma * 4;
  auto upto = [](int u) {
    const int n = (u * C::kLoads + kSlots - 1) / kSlots;
    return n < C::kLoads ? n : C::kLoads;
  };
  // One K step: its MFMAs, the fragment reads of the next step (step rstep of
  // the tile in stage st; with it the next tile's scales where rstep is 0) and
  // tile lt's loads from slot u0 on, in that interleaved order.
  auto kstep = [&](auto step, const uint8_t *st, int lt, int u0) {
    constexpr int kS = decltype(step)::value;
    constexpr int cb = kS & 1, nxt = cb ^ 1, rstep = (kS + 1) & 3;
    constexpr int kN = C::kMfma > C::kReads ? C::kMfma : C::kReads;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      if (i < C::kFN) {
        fa[nxt][i] = *reinterpret_cast<const v4i *>(st + a_base + i * kMx4PackedTile + rstep * 1024);
        if constexpr (rstep == 0) na[i] = *reinterpret_cast<const int *>(st + ea_base + i * 256);
      } else if (i < C::kReads) {
        const int g = i - C::kFN;
        fb[nxt][g] = *reinterpret_cast<const v4i *>(st + b_base + g * 32 * 128 + off_f[rstep]);
        if constexpr (rstep == 0) nb[g] = *reinterpret_cast<const int *>(st + eb_base + g * 256);
      }
      if (i < C::kMfma) {
        // one operand changes from MFMA to MFMA
        const int g = i / C::kFN, f = (g & 1) ? C::kFN - 1 - i % C::kFN : i % C::kFN;
        acc[f][g] = mfma_mx4<kS>(fa[cb][f], fb[cb][g], acc[f][g], ea[f], eb[g]);
#pragma unroll
        for (int j = 0; j < C::kLoads; ++j)
          if (j >= upto(u0 + i) && j < upto(u0 + i + 1)) issue_one(lt, j);
      }
    }
    constexpr int kMaskMfma = 0x008, kMaskVmemRead = 0x020, kMaskDsRead = 0x100;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      if (i < C::kReads) __builtin_amdgcn_sched_group_barrier(kMaskDsRead, rstep == 0 ? 2 : 1, 0);
      if (i < C::kMfma) {
        __builtin_amdgcn_sched_group_barrier(kMaskMfma, 1, 0);
#pragma unroll
        for (int j = 0; j < C::kLoads; ++j)
          if (j >= upto(u0 + i) && j < upto(u0 + i + 1))
            __builtin_amdgcn_sched_group_barrier(kMaskVmemRead, 1, 0);
      }
    }
  };

  // ---- main loop ------------------------------------------------------------
#pragma unroll
  for (int t = 0; t < S - 1; ++t)
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) issue_one(t, j);
  wait_vmcnt<(S - 2) * C::kLoads>();  // tile 0 has landed
  lds_barrier();
#pragma unroll
  for (int j = 0; j < C::kLoads; ++j)
    if (j < upto(C::kMfma)) issue_one(S - 1, j);
#pragma unroll
  for (int f = 0; f < C::kFN; ++f) {
    fa[0][f] = *reinterpret_cast<const v4i *>(smem + a_base + f * kMx4PackedTile);
    ea[f] = *reinterpret_cast<const int *>(smem + ea_base + f * 256);
  }
#pragma unroll
  for (int g = 0; g < C::kFM; ++g) {
    fb[0][g] = *reinterpret_cast<const v4i *>(smem + b_base + g * 32 * 128 + off_f[0]);
    eb[g] = *reinterpret_cast<const int *>(smem + eb_base + g * 256);
  }
  for (int kt = 0; kt < kn; ++kt) {
    const uint8_t *st = smem + (kt % S) * C::kStage;
    kstep(IntC<0>{}, st, kt + S - 1, C::kMfma);
    kstep(IntC<1>{}, st, kt + S - 1, 2 * C::kMfma);
    kstep(IntC<2>{}, st, kt + S - 1, 3 * C::kMfma);
    // This wave's reads of tile kt are done once lgkmcnt drains, tile kt+1 has
    // landed once at most S-2 younger tiles are in flight; after the barrier
    // tile kt's stage takes tile kt+S.  At kt = kn-1 the reads of "tile kn" are
    // unused.
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    wait_vmcnt<(S - 2) * C::kLoads>();
    lds_barrier();
    kstep(IntC<3>{}, smem + ((kt + 1) % S) * C::kStage, kt + S, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < C::kFN; ++f) ea[f] = na[f];
#pragma unroll
    for (int g = 0; g < C::kFM; ++g) eb[g] = nb[g];
  }
  wait_vmcnt<0>();                     // the trailing out-of-range tiles
  __builtin_amdgcn_s_waitcnt(0xC07F);  // this wave's last reads
  lds_barrier();                       // every wave is done with the ring
  if constexpr (PARTS) {
    v4f *dst = sums + (((int64_t)place.part * tiles_m + tm) * tiles_n + tn) * (BN * BM / 4) +
               wave * (C::kMfma * 256) + lane;
#pragma unroll
    for (int f = 0; f < C::kFN; ++f)
#pragma unroll
      for (int g = 0; g < C::kFM; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          dst[((f * C::kFM + g) * 4 + j) * 64] = v4f{acc[f][g][4 * j], acc[f][g][4 * j + 1],
                                                     acc[f][g][4 * j + 2], acc[f][g][4 * j + 3]};
  } else {
    mx4_epilogue<C::kFN, C::kFM>(smem, acc, bp, M, N, Y, n0 + wn * C::kTN,
                                 (int64_t)m0 + wm * C::kTM, wave, lane);
  }
}

template <int BN, int BM, int WN, int WM, int S, bool PARTS>
__global__ __launch_bounds__(64 * WN * WM, 1) void mx4_gemm_kernel(
    const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe, const uint8_t *__restrict__ Wp,
    const float *__restrict__ bp, int M, int N, int K, uint16_t *__restrict__ Y, int tiles_m,
    int tiles_n, int parts, v4f *__restrict__ sums) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Mx4Cfg<BN, BM, WN, WM, S>::kSmem];
  mx4_gemm_body<BN, BM, WN, WM, S, PARTS>(smem, Xc, Xe, Wp, bp, M, N, K, Y, tiles_m, tiles_n, parts,
                                          sums);
}

// Adds the parts' sums in their order and writes the outputs: the workgroup of a
// tile, its waves and their registers as in the kernel that made them.
template <int BN, int BM, int WN, int WM, int S>
__global__ __launch_bounds__(64 * WN * WM, 1) void mx4_join_kernel(
    const v4f *__restrict__ sums, const float *__restrict__ bp, int M, int N,
    uint16_t *__restrict__ Y, int tiles_m, int tiles_n, int parts) {
  using C = Mx4Cfg<BN, BM, WN, WM, S>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[C::kOut];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tm = blockIdx.x / tiles_n, tn = blockIdx.x % tiles_n;
  const v4f *src = sums + (int64_t)blockIdx.x * (BN * BM / 4) + wave * (C::kMfma * 256) + lane;
  const int64_t step = (int64_t)tiles_m * tiles_n * (BN * BM / 4);
  v16f acc[C::kFN][C::kFM];
#pragma unroll
  for (int f = 0; f < C::kFN; ++f)
#pragma unroll
    for (int g = 0; g < C::kFM; ++g) acc[f][g] = v16f{};
  for (int p = 0; p < parts; ++p, src += step)
#pragma unroll
    for (int f = 0; f < C::kFN; ++f)
#pragma unroll
      for (int g = 0; g < C::kFM; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const v4f v = src[((f * C::kFM + g) * 4 + j) * 64];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[f][g][4 * j + i] += v[i];
        }
  mx4_epilogue<C::kFN, C::kFM>(smem, acc, bp, M, N, Y, tn * BN + (wave % WN) * C::kTN,
                               (int64_t)tm * BM + (wave / WN) * C::kTM, wave, lane);
}

template <int BN, int BM, int WN, int WM, int S, bool SPLITS>
hipError_t launch_mx4_tile(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                           const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                           int parts, void *workspace, hipStream_t st) {
  const int tiles_m = (int)((M + BM - 1) / BM), tiles_n = (int)((N + BN - 1) / BN);
  const unsigned tiles = (unsigned)(tiles_m * tiles_n);
  if constexpr (SPLITS) {
    if (parts > 1) {
      v4f *sums = static_cast<v4f *>(workspace);
      mx4_gemm_kernel<BN, BM, WN, WM, S, true><<<tiles * parts, 64 * WN * WM, 0, st>>>(
          Xc, Xe, Wp, bp, (int)M, (int)N, (int)K, Y, tiles_m, tiles_n, parts, sums);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      mx4_join_kernel<BN, BM, WN, WM, S><<<tiles, 64 * WN * WM, 0, st>>>(
          sums, bp, (int)M, (int)N, Y, tiles_m, tiles_n, parts);
      return hipGetLastError();
    }
  }
  mx4_gemm_kernel<BN, BM, WN, WM, S, false><<<tiles, 64 * WN * WM, 0, st>>>(
      Xc, Xe, Wp, bp, (int)M, (int)N, (int)K, Y, tiles_m, tiles_n, 1, nullptr);
  return hipGetLastError();
}

// The tiles.  Their times are fitted to 360 random launches on MI355X (33 .. 8192
// tokens, 512 .. 28672 channels, K = 512 .. 36864) whose weights come from HBM:
// the tile they pick is 0.6 % over the fastest of these (52 % at worst, on a 4 us
// launch), 1.0 % over the fastest of nine shapes tried.
//
// `splits`: with a workspace, few tiles share K between up to 16 workgroups each
// (not more than one of them per CU), whose sums a second launch adds: 3.4 us more
// and 0.535 us per MB of sums (fitted likewise).  512 tokens x 9216, K = 36864 120
// us in 3 parts and 156 without; 128 x 9216 47 and 68; 256 x 5120, K = 20480 32
// and 39; 64 x 5120 17.2 and 22.1; where it would not pay it is not picked (128 x
// 4096, K = 4096 7.9 and, in 2 parts, 10.7).
struct Mx4Tile {
  int bn, bm, threads;
  bool splits;
  Mx4Time time;
};
constexpr Mx4Tile kTiles[] = {
    {256, 256, 512, true, {-0.485, 9.442, 1.175, 0.631}},
    {192, 256, 512, false, {-0.814, 10.617, 1.014, 0.377}},
    {256, 128, 512, false, {-0.314, 5.946, 0.929, 0.334}},
    {192, 128, 512, false, {0.606, 5.894, 0.814, 0.190}},
    {128, 128, 512, true, {1.111, 4.042, 0.422, 0.205}},
    {64, 128, 256, false, {1.034, 3.509, 0.343, 0.105}},
    {128, 64, 512, true, {1.126, 2.890, 0.352, 0.141}},
    {64, 64, 256, true, {2.539, 1.251, 0.295, -0.004}},
};
constexpr int kTileCount = sizeof(kTiles) / sizeof(kTiles[0]);
constexpr int kMaxParts = 16;
constexpr double kJoin = 3.39, kJoinPerByte = 0.535e-6;

int64_t tiles_of(const Mx4Tile &t, int64_t M, int64_t N) {
  return ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn);
}
// A launch takes fewer than 2^32 work-items: a tile whose grid does not fit is
// left out.  256 x 256 has the fewest and is always there.
bool fits(const Mx4Tile &t, int64_t M, int64_t N) {
  return tiles_of(t, M, N) * t.threads <= (int64_t)UINT32_MAX;
}

}  // namespace detail

using namespace detail;

bool mx4_gemm_fits(int64_t M, int64_t N) { return fits(kTiles[0], M, N); }

bool mx4_gemm_may_share(int64_t M, int64_t N, int64_t K) {
  return 2 * tiles_of(kTiles[0], M, N) <= device_cus() && mx4_tiles(K) >= 4;
}

Mx4Plan mx4_gemm_plan(int64_t M, int64_t N, int64_t K, bool with_workspace) {
  const int64_t cus = device_cus(), kt = mx4_tiles(K);
  Mx4Plan best{};
  for (int i = 0; i < kTileCount; ++i) {
    const Mx4Tile &t = kTiles[i];
    if (i > 0 && !fits(t, M, N)) continue;
    const int64_t tiles = tiles_of(t, M, N);
    for (int64_t parts = 1; parts <= kMaxParts; ++parts) {
      if (parts > 1 &&
          (!with_workspace || !t.splits || tiles * parts > cus || kt < 2 * parts))
        break;
      const int64_t bytes = parts > 1 ? tiles * parts * t.bn * t.bm * 4 : 0;
      double us = t.time.us(tiles * parts, (kt + parts - 1) / parts, cus);
      if (parts > 1) us += kJoin + kJoinPerByte * (double)bytes;
      if ((i == 0 && parts == 1) || us < best.us)
        best = Mx4Plan{i, t.bn, t.bm, (int)parts, (size_t)bytes, us};
    }
  }
  return best;
}

hipError_t launch_mx4_gemm(const Mx4Plan &plan, const uint8_t *Xc, const uint8_t *Xe,
                           const uint8_t *Wp, const float *bp, int64_t M, int64_t N, int64_t K,
                           uint16_t *Y, void *ws, hipStream_t st) {
  const int n = plan.parts;
  switch (plan.tile) {
    case 0: return launch_mx4_tile<256, 256, 4, 2, 2, true>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 1: return launch_mx4_tile<192, 256, 2, 4, 2, false>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 2: return launch_mx4_tile<256, 128, 4, 2, 2, false>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 3: return launch_mx4_tile<192, 128, 2, 4, 2, false>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 4: return launch_mx4_tile<128, 128, 4, 2, 4, true>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 5: return launch_mx4_tile<64, 128, 2, 2, 4, false>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    case 6: return launch_mx4_tile<128, 64, 4, 2, 4, true>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
    default: return launch_mx4_tile<64, 64, 2, 2, 4, true>(Xc, Xe, Wp, bp, M, N, K, Y, n, ws, st);
  }
}

}  // namespace ot
