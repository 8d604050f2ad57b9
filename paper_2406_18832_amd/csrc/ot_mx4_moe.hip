// A mixture-of-experts layer on MX4 weights for at most 64 tokens, in two
// launches.
//
//   p    = softmax over a token's top_k largest logits (ties to the lower expert)
//   g_j  = W1_e x + b1_e for its j-th expert e
//   h_j  = max(g_j, 0), or silu(gate) * up of g_j's two halves   (fp32)
//   y    = fp16(sum_j p_j (W2_e mx4(h_j) + b2_e))
//
// Bound by reading the weights of the experts that some token chose, each once.
//
// Kernel 1: a workgroup takes 32 hidden channels of one expert and the tokens
// that chose it (found from the logits by every workgroup for itself: counting
// the logits before the expert's own takes less than a launch would), runs fc1
// over H with its waves sharing the K tiles, then forms the activation and the
// MX4 block of each token's 32 channels, which go to the workspace as row
// m top_k + j.  Experts that nobody chose have workgroups that end at once; with
// fewer choices than experts the workgroups go by choice instead of by expert.
// One workgroup more writes down every token's experts and weights.
//
// Kernel 2: a workgroup takes 16 output channels and all tokens.  Its waves
// share out the K tiles of all chosen experts in one row, add p_j times each
// expert's product to their own fp32 sums in LDS, and the waves' sums meet in
// wave order: no atomics, so the result does not vary.
#include "ot_mx4_stream.h"

namespace ot {
namespace detail {

constexpr int kMoeWaves1 = 8, kMoeWaves2 = 16;

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

// The largest of a token's keys below `below` (0: none), over the wave.
__device__ __forceinline__ uint32_t moe_next(const uint16_t *__restrict__ l, int E, uint32_t below,
                                             int lane) {
  uint32_t best = 0;
  for (int e = lane; e < E; e += 64) {
    const uint32_t k = moe_key(l[e], e);
    if (k < below) best = max(best, k);
  }
  return wave_max_u32(best);
}

struct MoeWs {
  uint8_t *codes, *scales;  // hidden rows [M top_k][F / 2], [T][M top_k][8]
  int *expert;              // [M top_k], -1: none
  float *weight;            // [M top_k]
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

// Every token's experts and weights (one workgroup).
__device__ void moe_route(const MoeArgs &a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int m = wave; m < a.M; m += blockDim.x >> 6) {
    const uint16_t *l = a.logits + (int64_t)m * a.E;
    uint32_t key = 0xffffffffu;
    float most = 0.f, sum = 0.f, w = 0.f;
    int expert = -1;
    for (int j = 0; j < a.top_k; ++j) {
      key = moe_next(l, a.E, key, lane);
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
}

// The hidden rows of up to 16 MB of an expert's tokens, columns c0 .. of its
// list: fc1 over H, activation, MX4.
template <bool GLU, int MB>
__device__ __forceinline__ void moe_hidden(const MoeArgs &a, v4f *red, int e, int f, int c0,
                                           int count, const int *list, const int *rank_of) {
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
  mx4_stream<RB, MB, RB * MB == 8 ? 1 : 2>(acc, w, x, wave, tiles, kMoeWaves1, lane);
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) red[((wave * RB + i) * MB + j) * 64 + lane] = acc[i][j];
  __syncthreads();

  // activation and MX4: a quad of lanes to a token, 8 channels to a lane
  if (threadIdx.x >= MB * 64) return;
  const int col = threadIdx.x >> 2, q = threadIdx.x & 3;
  float g[RB / 2][8];
#pragma unroll
  for (int u = 0; u < RB / 2; ++u)  // (the gate's and) the value's 32 rows
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int i = 2 * u + (q >> 1), l = 16 * (2 * (q & 1) + v) + (col & 15);
      v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int wv = 0; wv < kMoeWaves1; ++wv)
        s += red[((wv * RB + i) * MB + (col >> 4)) * 64 + l];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t row = row0 + u * (int64_t)a.F + 8 * q + 4 * v + t;
        g[u][4 * v + t] = s[t] + (a.b1 ? a.b1[row] : 0.f);
      }
    }
  float h[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    if constexpr (GLU) {
      const float silu = g[0][t] / (1.f + expf(-g[0][t]));
      h[t] = silu * g[RB / 2 - 1][t];
    } else {
      h[t] = g[0][t] > 0.f || g[0][t] != g[0][t] ? g[0][t] : 0.f;  // keeps a NaN
    }
  }
  uint32_t most = abs_bits(h[0]);
#pragma unroll
  for (int t = 1; t < 8; ++t) most = max(most, abs_bits(h[t]));
  const uint32_t b = mx4_scale_byte(quad_max(most));
  const uint32_t codes = mx4_codes8(h, b);
  if (c0 + col >= count) return;
  const int m = list[c0 + col], rows = a.M * a.top_k;
  const int64_t slot = (int64_t)m * a.top_k + rank_of[m];
  *reinterpret_cast<uint32_t *>(a.ws.codes + slot * (a.F / 2) + 16 * f + 4 * q) = codes;
  if (q == 0) {
    a.ws.scales[((int64_t)(f >> 3) * rows + slot) * 8 + (f & 7)] = (uint8_t)b;
    // the last tile's scales past F
    if (f == a.F / 32 - 1)
      for (int i = f + 1; i & 7; ++i) a.ws.scales[((int64_t)(i >> 3) * rows + slot) * 8 + (i & 7)] = 0;
  }
}

// gridDim.x = F / 32 (+ 1: the routing), gridDim.y = min(E, M top_k).  An expert
// of more than 16 tokens takes 32 at a time (MB 2), reading its weights again for
// the second 32.
template <bool GLU, int MB>
__global__ __launch_bounds__(64 * kMoeWaves1) void moe_mx4_hidden_kernel(MoeArgs a) {
  __shared__ v4f red[kMoeWaves1 * (GLU ? 4 : 2) * MB * 64];
  __shared__ int first_of, list[64], rank_of[64];
  __shared__ unsigned long long members;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int f = blockIdx.x, hidden_tiles = a.F / 32;
  if (f == hidden_tiles) {
    if (blockIdx.y == 0) moe_route(a);
    return;
  }

  // ---- this workgroup's expert ------------------------------------------------
  int e = blockIdx.y;
  const bool by_choice = (int)gridDim.y < a.E;
  if (by_choice) {
    if (wave == 0) {
      const int m = blockIdx.y / a.top_k, j = blockIdx.y % a.top_k;
      uint32_t key = 0xffffffffu;
      for (int i = 0; i <= j; ++i) key = moe_next(a.logits + (int64_t)m * a.E, a.E, key, lane);
      if (lane == 0) first_of = moe_chosen(key) ? 0xffff - (int)(key & 0xffff) : -1;
    }
    __syncthreads();
    e = first_of;
    if (e < 0) return;
  }

  // ---- the tokens that chose it: 8 threads to a token count the logits before
  // the expert's own --------------------------------------------------------------
  {
    const int m = threadIdx.x >> 3, part = threadIdx.x & 7;
    bool in = false;
    int before = 0;
    if (m < a.M) {
      const uint16_t *l = a.logits + (int64_t)m * a.E;
      const uint32_t own = moe_key(l[e], e);
      for (int i = part; i < a.E; i += 8) before += moe_key(l[i], i) > own;
      in = moe_chosen(own);
    }
    before += __shfl_xor(before, 1);
    before += __shfl_xor(before, 2);
    before += __shfl_xor(before, 4);
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

  if (MB == 1 || count <= 16) {
    moe_hidden<GLU, 1>(a, red, e, f, 0, count, list, rank_of);
  } else {
    moe_hidden<GLU, MB>(a, red, e, f, 0, count, list, rank_of);
    if (count > 32) {
      __syncthreads();  // the sums of the first 32 are read
      moe_hidden<GLU, MB>(a, red, e, f, 32, count, list, rank_of);
    }
  }
}

// One expert's K tiles t0 .. t1-1 for this wave: p_j times the product onto the
// wave's sums.
template <int MB>
__device__ __forceinline__ void moe_expert(const MoeArgs &a, const Mx4Rows<1> &w,
                                           const Mx4Cols<1> &cols, const uint16_t *slots, int c0,
                                           int count, int t0, int t1, const float *weight,
                                           float *sums, int lane) {
  Mx4Cols<MB> x;
  x.codes = cols.codes;
  x.scales = cols.scales;
  x.scale_step = cols.scale_step;
  x.blocks = cols.blocks;
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const int c = c0 + 16 * j + (lane & 15);
    x.aim(j, c < count ? slots[c] : -1, a.F, lane);
  }
  v4f acc[1][MB];
#pragma unroll
  for (int j = 0; j < MB; ++j) acc[0][j] = v4f{0.f, 0.f, 0.f, 0.f};
  mx4_stream<1, MB, MB == 1 ? 3 : 1>(acc, w, x, t0, t1, 1, lane);
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const int c = c0 + 16 * j + (lane & 15);
    if (c < count) {
      const int slot = slots[c];
      v4f *s = reinterpret_cast<v4f *>(sums + (slot / a.top_k) * 16 + 4 * (lane >> 4));
      *s += weight[slot] * acc[0][j];
    }
  }
}

__global__ __launch_bounds__(64 * kMoeWaves2) void moe_mx4_out_kernel(MoeArgs a) {
  // LDS: the waves' sums [waves][M][16], the slots' weights and experts, each
  // expert's tokens as a mask and its slots in token order, the chosen experts
  extern __shared__ v4f lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nslots = a.M * a.top_k;
  float *sums = reinterpret_cast<float *>(lds);
  unsigned long long *mask = reinterpret_cast<unsigned long long *>(sums + kMoeWaves2 * a.M * 16);
  float *weight = reinterpret_cast<float *>(mask + a.E);
  int *expert = reinterpret_cast<int *>(weight + nslots);
  uint16_t *slots = reinterpret_cast<uint16_t *>(expert + nslots);  // [E][M]
  uint16_t *chosen = slots + a.E * a.M;                             // [E]
  __shared__ int nchosen;

  for (int i = threadIdx.x; i < kMoeWaves2 * a.M * 16; i += blockDim.x) sums[i] = 0.f;
  for (int i = threadIdx.x; i < a.E; i += blockDim.x) mask[i] = 0;
  for (int i = threadIdx.x; i < nslots; i += blockDim.x) {
    weight[i] = a.ws.weight[i];
    expert[i] = a.ws.expert[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nslots; i += blockDim.x)
    if (expert[i] >= 0) atomicOr(&mask[expert[i]], 1ull << (i / a.top_k));
  __syncthreads();
  for (int i = threadIdx.x; i < nslots; i += blockDim.x) {
    const int e = expert[i];
    if (e >= 0)
      slots[e * a.M + __popcll(mask[e] & ((1ull << (i / a.top_k)) - 1))] = (uint16_t)i;
  }
  if (wave == 0) {
    int n = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const bool in = e0 + lane < a.E && mask[e0 + lane] != 0;
      const unsigned long long all = __ballot(in);
      if (in) chosen[n + __popcll(all & ((1ull << lane) - 1))] = (uint16_t)(e0 + lane);
      n += __popcll(all);
    }
    if (lane == 0) nchosen = n;
  }
  __syncthreads();

  // ---- this wave's share of the chosen experts' K tiles -----------------------------
  const int tiles = (a.F + kMx4Tile - 1) / kMx4Tile;
  const int total = __builtin_amdgcn_readfirstlane(nchosen) * tiles;
  const int i0 = (int)((int64_t)total * wave / kMoeWaves2);
  const int i1 = (int)((int64_t)total * (wave + 1) / kMoeWaves2);
  const int64_t blocks = (int64_t)a.E * a.H / 32;
  Mx4Cols<1> cols;
  cols.open(a.ws.codes, a.ws.scales, nslots, a.F);
  for (int i = i0; i < i1;) {
    const int n = i / tiles, t0 = i - n * tiles, t1 = min(tiles, t0 + i1 - i);
    const int e = __builtin_amdgcn_readfirstlane((int)chosen[n]);
    const int count = __builtin_amdgcn_readfirstlane(__popcll(mask[e]));
    Mx4Rows<1> w;
    w.aim(a.W2, blocks, tiles, (int64_t)e * a.H / 16 + blockIdx.x, lane);
    float *own = sums + wave * a.M * 16;
    if (count <= 16)
      moe_expert<1>(a, w, cols, slots + e * a.M, 0, count, t0, t1, weight, own, lane);
    else
      for (int c = 0; c < count; c += 32)
        moe_expert<2>(a, w, cols, slots + e * a.M, c, count, t0, t1, weight, own, lane);
    i += t1 - t0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.M * 4; i += blockDim.x) {
    const int m = i >> 2;
    const int64_t n = (int64_t)blockIdx.x * 16 + 4 * (i & 3);
    v4f s = v4f{0.f, 0.f, 0.f, 0.f};
    for (int v = 0; v < kMoeWaves2; ++v) s += lds[(v * a.M + m) * 4 + (i & 3)];
    if (a.b2)
      for (int j = 0; j < a.top_k; ++j) {
        const int e = expert[m * a.top_k + j];
        if (e >= 0)
          s += weight[m * a.top_k + j] *
               *reinterpret_cast<const v4f *>(a.b2 + (int64_t)e * a.H + n);
      }
    uint2 h;
    h.x = (uint32_t)float_to_half_bits(s[0]) | ((uint32_t)float_to_half_bits(s[1]) << 16);
    h.y = (uint32_t)float_to_half_bits(s[2]) | ((uint32_t)float_to_half_bits(s[3]) << 16);
    *reinterpret_cast<uint2 *>(a.Y + (int64_t)m * a.H + n) = h;
  }
}

size_t moe_out_lds(int M, int E, int top_k) {
  return (size_t)kMoeWaves2 * M * 64 + (size_t)E * 8 + (size_t)M * top_k * 8 + (size_t)E * M * 2 +
         (size_t)E * 2;
}

size_t align16(size_t n) { return (n + 15) & ~size_t(15); }

}  // namespace detail

using namespace detail;

size_t moe_mx4_workspace_bytes(int64_t M, int64_t F, int64_t top_k) {
  const size_t slots = (size_t)M * top_k;
  return align16(slots * (F / 2)) + align16((size_t)mx4_tiles(F) * slots * 8) +
         align16(slots * sizeof(int)) + align16(slots * sizeof(float));
}

hipError_t launch_moe_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint16_t *logits,
                          const uint8_t *W1, const float *b1, const uint8_t *W2, const float *b2,
                          int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k, bool glu,
                          uint16_t *Y, void *workspace, hipStream_t st) {
  const size_t slots = (size_t)M * top_k;
  uint8_t *p = static_cast<uint8_t *>(workspace);
  MoeArgs a{Xc, Xe, logits, W1, W2, b1, b2, (int)M, (int)H, (int)F, (int)E, (int)top_k, Y, {}};
  a.ws.codes = p;
  p += align16(slots * (F / 2));
  a.ws.scales = p;
  p += align16((size_t)mx4_tiles(F) * slots * 8);
  a.ws.expert = reinterpret_cast<int *>(p);
  p += align16(slots * sizeof(int));
  a.ws.weight = reinterpret_cast<float *>(p);
  const dim3 grid((unsigned)(F / 32 + 1), (unsigned)(E < (int64_t)slots ? E : (int64_t)slots));
  const int threads = 64 * kMoeWaves1;
  if (M <= 16) {
    if (glu) moe_mx4_hidden_kernel<true, 1><<<grid, threads, 0, st>>>(a);
    else moe_mx4_hidden_kernel<false, 1><<<grid, threads, 0, st>>>(a);
  } else {
    if (glu) moe_mx4_hidden_kernel<true, 2><<<grid, threads, 0, st>>>(a);
    else moe_mx4_hidden_kernel<false, 2><<<grid, threads, 0, st>>>(a);
  }
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  moe_mx4_out_kernel<<<(unsigned)(H / 16), 64 * kMoeWaves2,
                       moe_out_lds((int)M, (int)E, (int)top_k), st>>>(a);
  return hipGetLastError();
}

}  // namespace ot
