// The MX4 linear above 64 tokens:  Y = fp16(sum_k x w + b'), both operands in
// MX4 (ot_mx4.h), products and scales on v_mfma_scale_f32_32x32x64_f8f6f4, sums
// in fp32.
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
#include "ot_mx4.h"

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
  static constexpr int kLoadsE = (BN + BM) / 32 / kWaves;                     // 256 bytes each
  static constexpr int kLoads = kLoadsA + kLoadsB + kLoadsE;
  static constexpr int kMfma = kFN * kFM, kReads = kFN + kFM;
  static constexpr int kOut = BN * BM * 2;  // the fp16 output tile, staged after the loop
  static constexpr int kSmem = S * kStage > kOut ? S * kStage : kOut;
  static_assert(kLoadsA * 8 * kWaves == BN && kLoadsB * 8 * kWaves == BM, "whole code loads");
  static_assert(kLoadsE * 32 * kWaves == BN + BM, "whole scale loads");
  static_assert(kTN % 32 == 0 && kTM % 32 == 0, "32x32 blocks");
  static_assert(S >= 2 && (S - 2) * kLoads <= 63, "vmcnt range");
  static_assert(kSmem <= 160 * 1024, "LDS");
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

template <int BN, int BM, int WN, int WM, int S>
__device__ __forceinline__ void mx4_gemm_body(
    uint8_t *smem, const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe,
    const uint8_t *__restrict__ Wp, const float *__restrict__ bp, int M, int N, int K,
    uint16_t *__restrict__ Y, int tiles_m, int tiles_n, int group_m) {
  using C = Mx4Cfg<BN, BM, WN, WM, S>;
  const int KB = K / 2;                      // bytes of a token row
  const int KT = (K + kMx4Tile - 1) / kMx4Tile;
  const int NB = (N + 31) / 32;              // 32-row blocks of the packed weights

  // ---- tile schedule: each XCD a contiguous range of tiles, walked in groups
  // of group_m token tiles (as the int8 prefill) ------------------------------
  const int nwg = gridDim.x, bid = blockIdx.x;
  const int xcd = bid & 7, local = bid >> 3;
  const int per = nwg >> 3, rem = nwg & 7;
  const int lid = (xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per) + local;
  const int group_size = group_m * tiles_n;
  const int first_m = (lid / group_size) * group_m;
  const int gm = min(tiles_m - first_m, group_m);
  const int tm = first_m + (lid % group_size) % gm;
  const int tn = (lid % group_size) / gm;
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
  // Load j of K tile kt into its stage.  Tiles past the end of K load zeros
  // (out of range) into stages that nobody reads, so that every iteration has
  // the same number of loads in flight.
  auto issue_one = [&](int kt, int j) {
    uint8_t *st = smem + (kt % S) * C::kStage;
    if (j < C::kLoadsA) {
      const int ja = j < C::kLoadsA ? j : 0;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc_a, (lds_void *)(st + (wave * C::kLoadsA + ja) * 1024), 16,
          kt < KT ? off_a[ja] + (uint32_t)kt * kMx4PackedTile : kOobOffset, 0, 0, 0);
    } else if (j < C::kLoadsA + C::kLoadsB) {
      const int jb = j >= C::kLoadsA && j < C::kLoadsA + C::kLoadsB ? j - C::kLoadsA : 0;
      const int k0 = kt * kMx4TileBytes;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc_b, (lds_void *)(st + C::kABytes + (wave * C::kLoadsB + jb) * 1024), 16,
          k0 + ck_b[jb] < KB ? off_b[jb] + (uint32_t)k0 : kOobOffset, 0, 0, 0);
    } else {
      // scales: 256-byte piece q, of 32 weight rows or 32 token rows
      const int q = wave * C::kLoadsE + (j - C::kLoadsA - C::kLoadsB);
      const int t = min(kt, KT - 1);
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
        const int f = i / C::kFM, g = i % C::kFM;
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
  for (int kt = 0; kt < KT; ++kt) {
    const uint8_t *st = smem + (kt % S) * C::kStage;
    kstep(IntC<0>{}, st, kt + S - 1, C::kMfma);
    kstep(IntC<1>{}, st, kt + S - 1, 2 * C::kMfma);
    kstep(IntC<2>{}, st, kt + S - 1, 3 * C::kMfma);
    // This wave's reads of tile kt are done once lgkmcnt drains, tile kt+1 has
    // landed once at most S-2 younger tiles are in flight; after the barrier
    // tile kt's stage takes tile kt+S.  At kt = KT-1 the reads of "tile KT" are
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

  // ---- epilogue: bias, fp16, whole token rows out through LDS -----------------
  // Lane l of a 32x32 block holds token l mod 32 and, in registers 4j..4j+3,
  // channels 8j + 4 (l / 32) .. +3.  The wave's kTM token rows of kTN channels
  // are staged with the 8-byte unit u of row r at unit u ^ h(r), which spreads
  // the lanes of a write over the banks.
  constexpr int kUnits = C::kTN / 4;
  constexpr int kSwz = kUnits % 16 == 0 ? 16 : 8;
  constexpr int kCpr = C::kTN / 8;
  static_assert(kUnits % kSwz == 0, "the swizzle permutes whole groups of units");
  auto stage_swz = [](int r) { return kSwz == 16 ? (r & 15) : ((r >> 1) & 7); };
  uint16_t *tile = reinterpret_cast<uint16_t *>(smem) + wave * (C::kTM * C::kTN);
  const int nw0 = n0 + wn * C::kTN, mw0 = m0 + wm * C::kTM;
#pragma unroll
  for (int f = 0; f < C::kFN; ++f)
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
      for (int g = 0; g < C::kFM; ++g) {
        const int r = g * 32 + fr;
        uint2 h;
        h.x = (uint32_t)float_to_half_bits(acc[f][g][4 * j] + b4.x) |
              ((uint32_t)float_to_half_bits(acc[f][g][4 * j + 1] + b4.y) << 16);
        h.y = (uint32_t)float_to_half_bits(acc[f][g][4 * j + 2] + b4.z) |
              ((uint32_t)float_to_half_bits(acc[f][g][4 * j + 3] + b4.w) << 16);
        *reinterpret_cast<uint2 *>(tile + r * C::kTN + 4 * ((nl >> 2) ^ stage_swz(r))) = h;
      }
    }
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_wave_barrier();
#pragma unroll 2
  for (int c0 = 0; c0 < C::kTM * kCpr; c0 += 64) {
    const int c = c0 + lane;
    const int r = c / kCpr, cc = c % kCpr;
    const int x = stage_swz(r);
    uint4 v = *reinterpret_cast<const uint4 *>(tile + r * C::kTN + (cc ^ (x >> 1)) * 8);
    if (x & 1) {  // the two 8-byte units of the pair are stored swapped
      const uint32_t t0 = v.x, t1 = v.y;
      v.x = v.z; v.y = v.w; v.z = t0; v.w = t1;
    }
    const int64_t m = mw0 + r;
    const int n = nw0 + cc * 8;
    if (m < M) {
      uint16_t *dst = Y + m * (int64_t)N + n;
      if ((N & 7) == 0 && n + 7 < N) {
        *reinterpret_cast<uint4 *>(dst) = v;
      } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        for (int i = 0; i < 8; ++i)
          if (n + i < N) dst[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}

template <int BN, int BM, int WN, int WM, int S>
__global__ __launch_bounds__(64 * WN * WM, 1) void mx4_gemm_kernel(
    const uint8_t *__restrict__ Xc, const uint8_t *__restrict__ Xe, const uint8_t *__restrict__ Wp,
    const float *__restrict__ bp, int M, int N, int K, uint16_t *__restrict__ Y, int tiles_m,
    int tiles_n, int group_m) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Mx4Cfg<BN, BM, WN, WM, S>::kSmem];
  mx4_gemm_body<BN, BM, WN, WM, S>(smem, Xc, Xe, Wp, bp, M, N, K, Y, tiles_m, tiles_n, group_m);
}

template <int BN, int BM, int WN, int WM, int S>
hipError_t launch_mx4_tile(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                           const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                           hipStream_t st) {
  const int tiles_m = (int)((M + BM - 1) / BM), tiles_n = (int)((N + BN - 1) / BN);
  mx4_gemm_kernel<BN, BM, WN, WM, S><<<(unsigned)(tiles_m * tiles_n), 64 * WN * WM, 0, st>>>(
      Xc, Xe, Wp, bp, (int)M, (int)N, (int)K, Y, tiles_m, tiles_n, 8);
  return hipGetLastError();
}

struct Mx4Tile {
  int bn, bm, threads;
  const char *name;
};
constexpr Mx4Tile kTiles[] = {{256, 256, 512, "prefill 256x256"},
                              {128, 128, 256, "prefill 128x128"},
                              {64, 64, 256, "prefill 64x64"}};

int64_t tiles_of(const Mx4Tile &t, int64_t M, int64_t N) {
  return ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn);
}
bool fits(const Mx4Tile &t, int64_t M, int64_t N) {
  return tiles_of(t, M, N) * t.threads <= (int64_t)UINT32_MAX;
}

int pick_tile(int64_t M, int64_t N, int64_t K) {
  (void)K;
  const int64_t cus = device_cus();
  if (tiles_of(kTiles[0], M, N) >= cus / 2 || !fits(kTiles[1], M, N)) return 0;
  if (tiles_of(kTiles[1], M, N) >= cus / 2 || !fits(kTiles[2], M, N)) return 1;
  return 2;
}

}  // namespace detail

using namespace detail;

bool mx4_gemm_fits(int64_t M, int64_t N) { return fits(kTiles[0], M, N); }

const char *mx4_gemm_tile_name(int64_t M, int64_t N, int64_t K) {
  return kTiles[pick_tile(M, N, K)].name;
}

hipError_t launch_mx4_gemm(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                           const float *bp, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                           hipStream_t st) {
  switch (pick_tile(M, N, K)) {
    case 0: return launch_mx4_tile<256, 256, 4, 2, 2>(Xc, Xe, Wp, bp, M, N, K, Y, st);
    case 1: return launch_mx4_tile<128, 128, 2, 2, 4>(Xc, Xe, Wp, bp, M, N, K, Y, st);
    default: return launch_mx4_tile<64, 64, 2, 2, 8>(Xc, Xe, Wp, bp, M, N, K, Y, st);
  }
}

}  // namespace ot
