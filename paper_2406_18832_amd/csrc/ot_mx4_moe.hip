// A mixture-of-experts layer on MX4 weights for at most 64 tokens, in two
// launches, or three where there are few output channels.
//
//   p    = softmax over a token's top_k largest logits (ties to the lower expert)
//   g_j  = W1_e x + b1_e for its j-th expert e
//   h_j  = max(g_j, 0), or silu(gate) * up of g_j's two halves   (fp32)
//   y    = fp16(sum_j p_j (W2_e mx4(h_j) + b2_e))
//
// Bound by reading the weights of the experts that some token chose, each once.
//
// Kernel 1: a workgroup serves one expert and the tokens that chose it (found
// from the logits by every workgroup for itself: counting the logits before the
// expert's own takes less than a launch would).  A wave runs fc1 over H for 32
// hidden channels (or, where there are few, shares the K tiles with others), then
// forms the activation and the MX4 block of each token's 32 channels, which go to
// the workspace in the operand order of the other kernel.  Experts that nobody
// chose have workgroups that end at once; with fewer choices than experts the
// workgroups go by choice instead of by expert.  A row of workgroups more writes
// down every token's experts and weights.
//
// Kernel 2: a workgroup takes 16 output channels and all tokens.  Its waves
// share out the K tiles of all chosen experts in one row, add p_j times each
// expert's product to their own fp32 sums in LDS, and the waves' sums meet in
// wave order: no atomics, so the result does not vary.  Where H / 16 workgroups
// leave CUs idle, several share that row of K tiles, and kernel 3 adds their sums.
#include "ot_mx4_stream.h"

namespace ot {
namespace detail {

constexpr int kMoeWaves1 = 4, kMoeWaves2 = 16;

__device__ __forceinline__ uint2 half4(v4f s) {
  uint2 h;
  h.x = (uint32_t)float_to_half_bits(s[0]) | ((uint32_t)float_to_half_bits(s[1]) << 16);
  h.y = (uint32_t)float_to_half_bits(s[2]) | ((uint32_t)float_to_half_bits(s[3]) << 16);
  return h;
}

// A token's logit for expert e as an integer that orders as the choice does:
// larger comes first, the lower expert first among equals, -0 equal to 0, NaN
// after every number.
__device__ __forceinline__ uint32_t moe_key(uint16_t l, int e) {
  uint32_t k;
  if ((l & 0x7fff) > 0x7c00) k = 0;
  else if ((l & 0x7fff) == 0) k = 0x8000;
  else k = (l & 0x8000) ? (uint16_t)~l : l | 0x8000u;
  return k << 16 | (0xffffu - (uint32_t)e);
}
// Keys of -inf and NaN: an expert with such a logit is not chosen.
__device__ __forceinline__ bool moe_chosen(uint32_t key) { return key >> 16 > 0x03ff; }
__device__ __forceinline__ float moe_logit(uint32_t key) {
  const uint32_t k = key >> 16;
  return half_bits_to_float((uint16_t)(k & 0x8000 ? k & 0x7fff : ~k));
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off));
  return v;
}

// A token's keys over a wave, OT_MOE_MAX_EXPERTS / 64 to a lane (0: no expert).
struct MoeKeys {
  static constexpr int kLane = OT_MOE_MAX_EXPERTS / 64;
  uint32_t k[kLane];
  __device__ __forceinline__ MoeKeys(const uint16_t *__restrict__ l, int E, int lane) {
#pragma unroll
    for (int i = 0; i < kLane; ++i) {
      const int e = 64 * i + lane;
      k[i] = e < E ? moe_key(l[e], e) : 0;
    }
  }
  // the largest key below `below` (0: none)
  __device__ __forceinline__ uint32_t next(uint32_t below) const {
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < kLane; ++i)
      if (k[i] < below) best = max(best, k[i]);
    return wave_max_u32(best);
  }
};

// Hidden rows.  An expert's tokens in order take columns 0, 1, ..; with G =
// ceil(M / 16) and T = ceil(F / 256), columns 16 g .. +15 of expert e are
//   codes  [e G + g][T][2 instructions][64 lanes][16 bytes]
//   scales [e G + g][T][64 lanes][4 bytes]  (bytes 0 and 2: instructions 0 and 1)
// as v_mfma_scale_f32_16x16x128_f8f6f4 takes them (ot_mx4_stream.h), so that the
// other kernel's loads are whole KiB.  Row by row, those loads (32 bytes from each
// of 16 rows) took longer than its weights'.  Most of it is never touched.  It is
// 2304 G T bytes an expert: for F a multiple of 256 8.5 G / H of the weights of ReLU
// experts (0.2 % of them at H = 4096 and up to 16 tokens) and two thirds of that of
// gated ones, else more.
struct MoeWs {
  uint8_t *codes, *scales;
  int *expert;              // [M top_k], -1: none
  float *weight;            // [M top_k]
  float *sums;              // [parts][M][H], with more than one part
};

struct MoeArgs {
  const uint8_t *Xc, *Xe;
  const uint16_t *logits;
  const uint8_t *W1, *W2;
  const float *b1, *b2;
  int M, H, F, E, top_k;
  uint16_t *Y;
  MoeWs ws;
};

// Token m's experts and weights, by one wave.
__device__ __forceinline__ void moe_route(const MoeArgs &a, int m, int lane) {
  const MoeKeys keys(a.logits + (int64_t)m * a.E, a.E, lane);
  uint32_t key = 0xffffffffu;
  float most = 0.f, sum = 0.f, w = 0.f;
  int expert = -1;
  for (int j = 0; j < a.top_k; ++j) {
    key = keys.next(key);
    if (!moe_chosen(key)) break;
    const float v = moe_logit(key);
    if (j == 0) most = v;
    const float x = v == most ? 1.f : expf(v - most);
    sum += x;
    if (lane == j) {
      w = x;
      expert = 0xffff - (int)(key & 0xffff);
    }
  }
  if (lane < a.top_k) {
    a.ws.expert[m * a.top_k + lane] = expert;
    a.ws.weight[m * a.top_k + lane] = expert < 0 ? 0.f : w / sum;
  }
}

// The hidden channels 32 f .. +31 of up to 16 MB of an expert's tokens (columns c0
// .. of its list): fc1 over H by this wave, or its share `part` of `parts` waves'
// K tiles, whose sums meet in red; activation; MX4.
template <bool GLU, int MB>
__device__ __forceinline__ void moe_hidden(const MoeArgs &a, v4f *red, int part, int parts, int e,
                                           int f, int c0, int count, const int *list) {
  constexpr int RB = GLU ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t F1 = GLU ? 2 * (int64_t)a.F : a.F;
  const int64_t blocks = a.E * F1 / 32;
  const int tiles = (a.H + kMx4Tile - 1) / kMx4Tile;
  const int64_t row0 = e * F1 + 32 * (int64_t)f;
  Mx4Rows<RB> w;
  {
    Mx4Rows<2> half;
    half.aim(a.W1, blocks, tiles, row0 / 16, lane);
    w.scale_step = half.scale_step;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w.codes[i] = half.codes[i];
      w.scales[i] = half.scales[i];
    }
    if constexpr (GLU) {
      half.aim(a.W1, blocks, tiles, (row0 + a.F) / 16, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        w.codes[2 + i] = half.codes[i];
        w.scales[2 + i] = half.scales[i];
      }
    }
  }
  Mx4Cols<MB> x;
  x.open(a.Xc, a.Xe, a.M, a.H);
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const int c = c0 + 16 * j + (lane & 15);
    x.aim(j, c < count ? list[c] : -1, a.H, lane);
  }
  v4f acc[RB][MB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  mx4_stream<RB, MB, RB * MB == 8 ? 1 : 2>(acc, w, x, part, tiles, parts, lane);
  if (parts > 1) {  // the same for the whole workgroup
    __syncthreads();  // an earlier call's sums are read
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < MB; ++j) red[((wave * RB + i) * MB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    if (part > 0) return;
    for (int v = 1; v < parts; ++v)
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[i][j] += red[(((wave + v) * RB + i) * MB + j) * 64 + lane];
  }
  if (f >= a.F / 32) return;  // a wave past the last channels

  // Lane l holds, for column l mod 16, rows 4 (l / 16) .. +3 of each unit: eight
  // channels of the token's block, whose four lanes are 16 apart.
  const int q = lane >> 4;
  const int64_t b_at = row0 + 4 * q;
  float b1[RB][4];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const float4 v = a.b1 ? *reinterpret_cast<const float4 *>(a.b1 + b_at + (i >> 1) * (int64_t)a.F +
                                                             16 * (i & 1))
                          : make_float4(0.f, 0.f, 0.f, 0.f);
    b1[i][0] = v.x; b1[i][1] = v.y; b1[i][2] = v.z; b1[i][3] = v.w;
  }
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    float h[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int u = t >> 2, r = t & 3;
      const float g = acc[u][j][r] + b1[u][r];
      if constexpr (GLU) {
        const float up = acc[RB / 2 + u][j][r] + b1[RB / 2 + u][r];
        h[t] = g / (1.f + expf(-g)) * up;
      } else {
        h[t] = g > 0.f || g != g ? g : 0.f;  // keeps a NaN
      }
    }
    uint32_t most = abs_bits(h[0]);
#pragma unroll
    for (int t = 1; t < 8; ++t) most = max(most, abs_bits(h[t]));
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const uint32_t b = mx4_scale_byte(most);
    const uint32_t codes = mx4_codes8(h, b);
    const int c = c0 + 16 * j + (lane & 15);
    if (c >= count) continue;
    // block f of the row is block 4 hf + st of K tile f / 8: instruction st / 2,
    // lane group hf + 2 (st mod 2)
    const int64_t group = (int64_t)e * ((a.M + 15) / 16) + (c >> 4), tiles2 = (a.F + 255) / 256;
    auto lane_of = [&](int blk) { return 16 * ((blk >> 2) + 2 * (blk & 1)) + (c & 15); };
    const int blk = f & 7;
    uint16_t *dst = reinterpret_cast<uint16_t *>(
        a.ws.codes + (group * tiles2 + (f >> 3)) * 2048 + (blk >> 1 & 1) * 1024 +
        lane_of(blk) * 16 + 2 * q);
    dst[0] = (uint16_t)codes;
    dst[4] = (uint16_t)(codes >> 16);
    if (q == 0) {
      uint8_t *sc = a.ws.scales + (group * tiles2 + (f >> 3)) * 256;
      sc[lane_of(blk) * 4 + (blk & 2)] = (uint8_t)b;
      if (f == a.F / 32 - 1)  // the last tile's scales past F: a finite one, against zeros
        for (int i = blk + 1; i < 8; ++i) sc[lane_of(i) * 4 + (i & 2)] = 0;
    }
  }
}

// gridDim.x = 1 (the routing) + groups of hidden blocks, gridDim.y = min(E, M top_k).
// A workgroup's waves take kMoeWaves1 / parts blocks of 32 hidden channels, `parts`
// waves each.  An expert of more than 16 tokens takes 32 at a time (MB 2), reading
// its weights again for the second 32.  MI355X: one token through two of eight experts
// of 16384, H = 4096 16.2 us (4.4 TB/s of weights); 64 through 32 gated ones of 1408,
// H = 2048 22.3 (4.4 TB/s).
template <bool GLU, int MB>
__global__ __launch_bounds__(64 * kMoeWaves1, 2) void moe_mx4_hidden_kernel(MoeArgs a, int parts) {
  extern __shared__ v4f red[];  // parts > 1: [waves][RB][MB][64]
  __shared__ int first_of, list[64], rank_of[64];
  __shared__ unsigned long long members;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0) {  // first, since the other kernel waits for it: the routing
    for (int m = blockIdx.y * kMoeWaves1 + wave; m < a.M; m += gridDim.y * kMoeWaves1)
      moe_route(a, m, lane);
    return;
  }

  // ---- this workgroup's expert ------------------------------------------------
  int e = blockIdx.y;
  const bool by_choice = (int)gridDim.y < a.E;
  if (by_choice) {
    if (wave == 0) {
      const int m = blockIdx.y / a.top_k, j = blockIdx.y % a.top_k;
      const MoeKeys keys(a.logits + (int64_t)m * a.E, a.E, lane);
      uint32_t key = 0xffffffffu;
      for (int i = 0; i <= j; ++i) key = keys.next(key);
      if (lane == 0) first_of = moe_chosen(key) ? 0xffff - (int)(key & 0xffff) : -1;
    }
    __syncthreads();
    e = first_of;
    if (e < 0) return;
  }

  // ---- the tokens that chose it: a few threads to a token count the logits before
  // the expert's own --------------------------------------------------------------
  {
    constexpr int kShare = kMoeWaves1;  // 64 tokens
    const int m = threadIdx.x / kShare, part = threadIdx.x % kShare;
    bool in = false;
    int before = 0;
    if (m < a.M) {
      const uint16_t *l = a.logits + (int64_t)m * a.E;
      const uint32_t own = moe_key(l[e], e);
      for (int i0 = part; i0 < a.E; i0 += 8 * kShare) {  // 8 loads at a time
        uint16_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = l[min(i0 + u * kShare, a.E - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = i0 + u * kShare;
          before += i < a.E && moe_key(v[u], i) > own;
        }
      }
      in = moe_chosen(own);
    }
#pragma unroll
    for (int off = 1; off < kShare; off <<= 1) before += __shfl_xor(before, off);
    if (part == 0) rank_of[m] = in && before < a.top_k ? before : -1;
  }
  __syncthreads();
  if (wave == 0) {
    const unsigned long long all = __ballot(rank_of[lane] >= 0);
    if (lane == 0) members = all;
    if (rank_of[lane] >= 0) list[__popcll(all & ((1ull << lane) - 1))] = lane;
  }
  __syncthreads();
  const unsigned long long all = members;
  if (all == 0) return;
  // by choice: the first token that chose the expert does its work
  if (by_choice && __builtin_ctzll(all) != (int)blockIdx.y / a.top_k) return;
  const int count = __builtin_amdgcn_readfirstlane(__popcll(all));

  const int part = wave % parts;
  const int f = (blockIdx.x - 1) * (kMoeWaves1 / parts) + wave / parts;
  if (parts == 1 && f >= a.F / 32) return;  // (otherwise the workgroup meets at barriers)
  if (MB == 1 || count <= 16) {
    moe_hidden<GLU, 1>(a, red, part, parts, e, f, 0, count, list);
  } else {
    for (int c0 = 0; c0 < count; c0 += 32)
      moe_hidden<GLU, MB>(a, red, part, parts, e, f, c0, count, list);
  }
}

// MB column blocks of 16 tokens to a step (an expert's further tokens are steps
// of their own, which read its weights again).  MI355X, as above: 15.9 us (4.5 TB/s),
// and 14.8 in two parts of 128 workgroups (3.3 TB/s), whose sums take 4.5 more.
template <int MB>
__global__ __launch_bounds__(64 * kMoeWaves2) void moe_mx4_out_kernel(MoeArgs a) {
  // LDS: the waves' sums and the biases' [waves + 1][M][16], the slots' weights and experts, each
  // expert's tokens as a mask and its slots in token order, the groups of up to
  // 16 MB tokens of the chosen experts (expert and first column)
  extern __shared__ v4f lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nslots = a.M * a.top_k;
  float *sums = reinterpret_cast<float *>(lds);
  unsigned long long *mask = reinterpret_cast<unsigned long long *>(sums + (kMoeWaves2 + 1) * a.M * 16);
  float *weight = reinterpret_cast<float *>(mask + a.E);
  int *expert = reinterpret_cast<int *>(weight + nslots);
  int *groups = expert + nslots;                                   // [<= E + nslots / 16]
  uint16_t *slots = reinterpret_cast<uint16_t *>(groups + a.E + nslots / 16);  // [E][M]
  __shared__ int ngroups;

  for (int i = threadIdx.x; i < kMoeWaves2 * a.M * 4; i += blockDim.x)
    lds[i] = v4f{0.f, 0.f, 0.f, 0.f};
  for (int i = threadIdx.x; i < a.E; i += blockDim.x) mask[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < nslots; i += blockDim.x) {
    const int e = a.ws.expert[i];
    expert[i] = e;
    weight[i] = a.ws.weight[i];
    if (e >= 0) atomicOr(&mask[e], 1ull << (i / a.top_k));
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nslots; i += blockDim.x) {
    const int e = expert[i];
    if (e >= 0)
      slots[e * a.M + __popcll(mask[e] & ((1ull << (i / a.top_k)) - 1))] = (uint16_t)i;
  }
  if (wave == 0) {
    int n = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const int mine = e0 + lane < a.E ? (__popcll(mask[e0 + lane]) + 16 * MB - 1) / (16 * MB) : 0;
      int sum = mine;  // inclusive prefix sum over the wave
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int other = __shfl_up(sum, off);
        if (lane >= off) sum += other;
      }
      for (int g = 0; g < mine; ++g)
        groups[n + sum - mine + g] = (e0 + lane) << 8 | g * 16 * MB;
      n += __shfl(sum, 63);
    }
    if (lane == 0) ngroups = n;
  }
  __syncthreads();

  // ---- this wave's share of the groups' K tiles, as one row of steps ------------------
  const int tiles = (a.F + kMx4Tile - 1) / kMx4Tile;
  const int total = __builtin_amdgcn_readfirstlane(ngroups) * tiles;
  // (at most 320 groups of 256 K tiles, and 2048 shares: 32 bits)
  int i0 = 0, i1 = total;
  if (gridDim.y > 1) {
    i0 = (int)((unsigned)total * blockIdx.y / gridDim.y);
    i1 = (int)((unsigned)total * (blockIdx.y + 1) / gridDim.y);
  }
  const int mine = i1 - i0;
  i1 = i0 + mine * (wave + 1) / kMoeWaves2;
  i0 += mine * wave / kMoeWaves2;
  const int64_t blocks = (int64_t)a.E * a.H / 32;
  float *own = sums + wave * a.M * 16;
  // Loads run kDepth steps ahead, over the groups' borders.
  struct Frag {
    v4i a[2], b[MB][2];
    uint32_t ea, eb[MB];
  };
  const int64_t per_expert = (a.M + 15) / 16;
  Mx4Rows<1> w;
  // (columns that no token takes are not loaded)
  const int64_t code_bytes = (int64_t)a.E * per_expert * tiles * 2048;
  const __amdgpu_buffer_rsrc_t rc = make_rsrc(a.ws.codes, (uint32_t)code_bytes);
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.ws.scales, (uint32_t)(code_bytes / 8));
  uint32_t xc[MB], xe[MB];  // this lane's bytes of K tile 0
  int aimed = -1;
  auto load = [&](Frag &f, int i) {
    const int g = i / tiles, t = i - g * tiles;
    if (g != aimed) {
      aimed = g;
      const int id = __builtin_amdgcn_readfirstlane(groups[g]);
      const int e = id >> 8, c0 = id & 255, count = __popcll(mask[e]);
      w.aim(a.W2, blocks, tiles, (int64_t)e * a.H / 16 + blockIdx.x, lane);
#pragma unroll
      for (int j = 0; j < MB; ++j) {
        const uint32_t group = (uint32_t)(e * per_expert + c0 / 16 + j);
        const bool in = c0 + 16 * j + (lane & 15) < count;
        xc[j] = in ? group * tiles * 2048 + lane * 16 : kOobOffset;
        xe[j] = in ? group * tiles * 256 + lane * 4 : kOobOffset;
      }
    }
    const v4i *p = reinterpret_cast<const v4i *>(w.codes[0] + (int64_t)t * kMx4PackedTile);
    f.a[0] = __builtin_nontemporal_load(p);
    f.a[1] = __builtin_nontemporal_load(p + 128);
    f.ea = *reinterpret_cast<const uint32_t *>(w.scales[0] + t * w.scale_step);
#pragma unroll
    for (int j = 0; j < MB; ++j) {  // (kOobOffset + t KiB stays out of range)
      f.b[j][0] = __builtin_bit_cast(
          v4i, __builtin_amdgcn_raw_buffer_load_b128(rc, xc[j] + t * 2048, 0, 0));
      f.b[j][1] = __builtin_bit_cast(
          v4i, __builtin_amdgcn_raw_buffer_load_b128(rc, xc[j] + t * 2048 + 1024, 0, 0));
      f.eb[j] = __builtin_amdgcn_raw_buffer_load_b32(rs, xe[j] + t * 256, 0, 0);
    }
  };
  v4f acc[MB];
#pragma unroll
  for (int j = 0; j < MB; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
  // p_j times the group's product onto the wave's sums
  auto flush = [&](int g) {
    const int id = __builtin_amdgcn_readfirstlane(groups[g]);
    const int e = id >> 8, c0 = id & 255, count = __popcll(mask[e]);
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      const int c = c0 + 16 * j + (lane & 15);
      if (c < count) {
        const int slot = slots[e * a.M + c];
        v4f *s = reinterpret_cast<v4f *>(own + (slot / a.top_k) * 16 + 4 * (lane >> 4));
        *s += weight[slot] * acc[j];
      }
      acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
    }
  };
  constexpr int kDepth = MB == 1 ? 4 : 2;
  Frag f[kDepth];
#pragma unroll
  for (int d = 0; d < kDepth; ++d)
    if (i0 + d < i1) load(f[d], i0 + d);
  // sum_j p_j b2_e meanwhile
  for (int i = threadIdx.x; i < a.M * 4; i += blockDim.x) {
    const int m = i >> 2;
    v4f s = v4f{0.f, 0.f, 0.f, 0.f};
    if (a.b2 && blockIdx.y == 0)
      for (int j = 0; j < a.top_k; ++j) {
        const int e = expert[m * a.top_k + j];
        if (e >= 0)
          s += weight[m * a.top_k + j] *
               *reinterpret_cast<const v4f *>(a.b2 + (int64_t)e * a.H + blockIdx.x * 16 +
                                              4 * (i & 3));
      }
    lds[(kMoeWaves2 * a.M + m) * 4 + (i & 3)] = s;
  }
  for (int i = i0; i < i1; i += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (i + d < i1) {
        const uint32_t ea = f[d].ea >> (8 * (lane >> 5));
#pragma unroll
        for (int j = 0; j < MB; ++j)
          acc[j] = mfma_mx4_16<0>(f[d].a[0], f[d].b[j][0], acc[j], ea, f[d].eb[j]);
#pragma unroll
        for (int j = 0; j < MB; ++j)
          acc[j] = mfma_mx4_16<2>(f[d].a[1], f[d].b[j][1], acc[j], ea, f[d].eb[j]);
        if (i + d + kDepth < i1) load(f[d], i + d + kDepth);
        if ((i + d + 1) % tiles == 0 || i + d + 1 == i1) flush((i + d) / tiles);
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.M * 4; i += blockDim.x) {
    const int m = i >> 2;
    const int64_t n = (int64_t)blockIdx.x * 16 + 4 * (i & 3);
    v4f s = lds[m * 4 + (i & 3)];
    for (int v = 1; v <= kMoeWaves2; ++v) s += lds[(v * a.M + m) * 4 + (i & 3)];
    if (gridDim.y > 1)
      *reinterpret_cast<v4f *>(a.ws.sums + ((int64_t)blockIdx.y * a.M + m) * a.H + n) = s;
    else
      *reinterpret_cast<uint2 *>(a.Y + (int64_t)m * a.H + n) = half4(s);
  }
}

// Adds the parts' sums, in their order: four channels to a thread.
__global__ __launch_bounds__(256) void moe_mx4_join_kernel(const float *__restrict__ sums,
                                                           int64_t outputs, int parts,
                                                           uint16_t *__restrict__ Y) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= outputs) return;
  v4f s = *reinterpret_cast<const v4f *>(sums + i);
#pragma unroll 4
  for (int p = 1; p < parts; ++p) s += *reinterpret_cast<const v4f *>(sums + p * outputs + i);
  *reinterpret_cast<uint2 *>(Y + i) = half4(s);
}

// Parts that the second kernel's work is shared out to: as many as give every CU a
// workgroup, each wave at least two K tiles (counting one step of tokens per
// expert).  On MI355X, whole layers with and without: 20 tokens, H = 768, 43 experts
// of 9728 41 and 68 us; 57, 512, 13 of 9696 (top 7) 39 and 87; one token, 864, 9
// gated of 12448 (top 6) 38 and 48.  Two parts, weights from HBM, medians of 12 turns
// that differ by 0.5 %: over 43 random layers 0.78 to 1.006 of the time with one, the
// less the more K tiles a wave has; 48 tokens, 1696, 63 of 4160 (top 6) 105 and 134 us;
// 64, 2048, 32 gated of 1408 (top 4) 37.9 and 41.6; at the least, of four to five K tiles
// to a wave, one, 512, 20 of 2048 (top 8) 17.06 and 17.02; 3, 1792, 21 of 1952 (top 3)
// 17.06 and 16.97.
int moe_parts(int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k) {
  const int64_t slots = M * top_k, steps = (E < slots ? E : slots) * mx4_tiles(F);
  int64_t parts = device_cus() / (H / 16);
  if (parts > steps / (2 * kMoeWaves2)) parts = steps / (2 * kMoeWaves2);
  return parts < 2 ? 1 : (int)parts;
}

size_t moe_out_lds(int M, int E, int top_k) {
  return (size_t)(kMoeWaves2 + 1) * M * 64 + (size_t)E * 8 + (size_t)M * top_k * 8 +
         (size_t)(E + M * top_k / 16) * 4 + (size_t)E * M * 2;
}

size_t align16(size_t n) { return (n + 15) & ~size_t(15); }

}  // namespace detail

using namespace detail;

static size_t moe_code_bytes(int64_t M, int64_t F, int64_t E) {
  return (size_t)(E * ((M + 15) / 16)) * mx4_tiles(F) * 2048;
}

size_t moe_mx4_workspace_bytes(int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k) {
  const size_t slots = (size_t)M * top_k;
  const int parts = moe_parts(M, H, F, E, top_k);
  return moe_code_bytes(M, F, E) + moe_code_bytes(M, F, E) / 8 + align16(slots * sizeof(int)) +
         align16(slots * sizeof(float)) + (parts > 1 ? (size_t)parts * M * H * sizeof(float) : 0);
}

hipError_t launch_moe_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint16_t *logits,
                          const uint8_t *W1, const float *b1, const uint8_t *W2, const float *b2,
                          int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k, bool glu,
                          uint16_t *Y, void *workspace, hipStream_t st) {
  const size_t slots = (size_t)M * top_k;
  uint8_t *p = static_cast<uint8_t *>(workspace);
  MoeArgs a{Xc, Xe, logits, W1, W2, b1, b2, (int)M, (int)H, (int)F, (int)E, (int)top_k, Y, {}};
  a.ws.codes = p;
  p += moe_code_bytes(M, F, E);
  a.ws.scales = p;
  p += moe_code_bytes(M, F, E) / 8;
  a.ws.expert = reinterpret_cast<int *>(p);
  p += align16(slots * sizeof(int));
  a.ws.weight = reinterpret_cast<float *>(p);
  p += align16(slots * sizeof(float));
  a.ws.sums = reinterpret_cast<float *>(p);
  // Waves to a block of hidden channels: enough that a CU has some 70 KB of weights
  // in flight (4 waves of gate and value rows, 8 of one kind), as far as H has K
  // tiles for them.  One token through two experts of 16384, H = 4096: 18.6 us with
  // one wave, 15.7 with two; 64 tokens through 32 gated ones of 1408, H = 2048: 22.2
  // with one, 24.2 with two (a second round of workgroups).
  const int64_t rows = E < (int64_t)slots ? E : (int64_t)slots, hidden = F / 32;
  const int64_t enough = (glu ? 4 : 8) * (int64_t)device_cus();
  int parts = 1;
  while (parts < kMoeWaves1 && rows * hidden * parts < enough && 2 * parts <= mx4_tiles(H))
    parts *= 2;
  const int64_t per_wg = kMoeWaves1 / parts;
  const dim3 grid((unsigned)((hidden + per_wg - 1) / per_wg + 1), (unsigned)rows);
  const int threads = 64 * kMoeWaves1;
  const int units = (glu ? 4 : 2) * (M <= 16 ? 1 : 2);
  const size_t sums = parts > 1 ? (size_t)kMoeWaves1 * units * 1024 : 0;
  if (M <= 16) {
    if (glu) moe_mx4_hidden_kernel<true, 1><<<grid, threads, sums, st>>>(a, parts);
    else moe_mx4_hidden_kernel<false, 1><<<grid, threads, sums, st>>>(a, parts);
  } else {
    if (glu) moe_mx4_hidden_kernel<true, 2><<<grid, threads, sums, st>>>(a, parts);
    else moe_mx4_hidden_kernel<false, 2><<<grid, threads, sums, st>>>(a, parts);
  }
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const size_t lds = moe_out_lds((int)M, (int)E, (int)top_k);
  const int out_parts = moe_parts(M, H, F, E, top_k);
  const dim3 out_grid((unsigned)(H / 16), (unsigned)out_parts);
  // 32 tokens of an expert to a step where it has more than 12 on average: with
  // fewer, half of the token loads and products would be of nobody
  if (M <= 16 || (int64_t)slots <= 12 * E)
    moe_mx4_out_kernel<1><<<out_grid, 64 * kMoeWaves2, lds, st>>>(a);
  else
    moe_mx4_out_kernel<2><<<out_grid, 64 * kMoeWaves2, lds, st>>>(a);
  err = hipGetLastError();
  if (err != hipSuccess || out_parts == 1) return err;
  const int64_t outputs = M * H;
  moe_mx4_join_kernel<<<(unsigned)((outputs / 4 + 255) / 256), 256, 0, st>>>(a.ws.sums, outputs,
                                                                             out_parts, Y);
  return hipGetLastError();
}

}  // namespace ot
