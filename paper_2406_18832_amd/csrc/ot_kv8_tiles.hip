// Attention over the 8-bit cache for many query rows (prompts, pieces of prompts):
// bound by the matrix cores.
//
// A workgroup takes 128 query rows (tokens times the query heads of one key head)
// of a sequence, 32 to each of its four waves, and goes over the pages that they
// see.  A page's codes are turned to fp16 once, on their way into LDS, where all
// waves read them as the A operands of v_mfma_f32_32x32x16_f16.
//
// S^T = K Q^T: lane l has query row l mod 32; K's row 8 a + 4 h + i of a tile of 32
// tokens is token 16 (a / 2) + 8 h + 4 (a mod 2) + i, so that the 16 results of a lane
// (h = l / 32; a, i) are the weights of two runs of eight tokens, each the lane's part
// of the B operand of one product O^T += V^T P^T.
#include <math.h>

#include "ot_kv8_attn.h"

namespace ot {
namespace detail {

constexpr int kTileWaves = 4, kTileRows = 32 * kTileWaves;

template <int DP>
__global__ __launch_bounds__(64 * kTileWaves) void kv8_tile_kernel(Kv8Attn a) {
  constexpr int kThreads = 64 * kTileWaves;
  constexpr int kKStride = DP + 8, kVStride = kKv8Page + 8;  // halves; off the banks
  constexpr int kSteps = DP / 16, kOut = DP / 32;
  constexpr int kUnits = DP * kKv8Page / 16;     // 16 bytes each, of K as of V
  constexpr int kLoads = 2 * kUnits / kThreads;  // K's units, then V's
  static_assert(kLoads * kThreads == 2 * kUnits && kUnits % 64 == 0, "a page in whole loads");
  __shared__ _Float16 ks[kKv8Page * kKStride];
  __shared__ _Float16 vs[DP * kVStride];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int h = blockIdx.x % a.Hkv;
  const int64_t slot = blockIdx.x / a.Hkv;
  const int G = a.Hq / a.Hkv;
  const int b = kv8_find(a.B, lane, slot,
                         [&](int i) { return kv8_tile_slot((int64_t)a.cu[i] * G, i, kTileRows); });
  if (b < 0) return;
  const Kv8Rows rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
  // counted from the end: under a causal mask the last tile has the most pages
  const int64_t tiles = ((int64_t)rows.n * G + kTileRows - 1) / kTileRows;
  const int64_t tile = tiles - 1 - (slot - kv8_tile_slot((int64_t)a.cu[b] * G, b, kTileRows));
  if (tile < 0 || tile >= tiles) return;
  const int64_t len0 = a.kv_len[b];
  const int len = (int)kv8_len(len0, a.cache.max_pages);
  const bool bad = len0 > len;
  const int row0 = (int)tile * kTileRows + 32 * wave;
  const int all = rows.n * G;
  const int first = (int)tile * kTileRows / G;
  const int last = min((int)(tile + 1) * kTileRows - 1, all - 1) / G;
  const Kv8Span span = kv8_span(len, rows.n, first, last - first + 1, a.causal, a.window);

  // this lane's query row
  const int row = row0 + col;
  const bool in = row < all;
  const int qi = (in ? row : all - 1) / G, head = h * G + (in ? row : all - 1) % G;
  const uint16_t *qp = a.q + (int64_t)(rows.row0 + qi) * a.ldq + head * a.D;
  v8h q[kSteps];
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    const int d = 16 * st + 8 * half;
    v4u w = {0u, 0u, 0u, 0u};
    if (d < a.D) w = *reinterpret_cast<const v4u *>(qp + d);
    q[st] = __builtin_bit_cast(v8h, w);
  }
  const int pos = len - rows.n + qi;
  const int key_hi = a.causal ? pos : len - 1;
  const int key_lo = a.window > 0 ? max(0, (int)kv8_max(pos - a.window + 1, 0)) : 0;
  // keys that every row of the wave sees
  const int wave_first = min(row0, all - 1) / G, wave_last = min(row0 + 31, all - 1) / G;
  const int all_hi = a.causal ? len - rows.n + wave_first : len - 1;
  const int all_lo = a.window > 0 ? (int)kv8_max(0, len - rows.n + wave_last - a.window + 1) : 0;

  float m = kNegInf, l = 0.f;
  v16f o[kOut];
#pragma unroll
  for (int t = 0; t < kOut; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  const float fac = a.scale * kLog2e;

  v4u code[kLoads];
  float f = 0.f, lg = 0.f, iv = 1.f;
  auto fetch = [&](int p) {
    int64_t page = kv8_page(a.cache.table, b, p, a.cache.max_pages, a.cache.num_pages);
    const bool none = page < 0 || bad;
    if (page < 0) page = 0;
    const int64_t ph = page * a.Hkv + h;
    const uint8_t *kp = a.cache.Kc + ph * (DP * kKv8Page), *vp = a.cache.Vc + ph * (DP * kKv8Page);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * kThreads + tid;
      code[u] = *reinterpret_cast<const v4u *>(at < kUnits ? kp + at * 16 : vp + (at - kUnits) * 16);
    }
    f = none ? __builtin_nanf("") : a.cache.Ks[ph] * fac;
    value_scale(none ? 0.f : a.cache.Vs[ph], lg, iv);
  };
  if (span.p0 < span.p1) fetch(span.p0);

  for (int p = span.p0; p < span.p1; ++p) {
    __syncthreads();  // the page before is done with
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = (u * kThreads + tid) * 16, vat = at - 16 * kUnits;
      _Float16 *to = at < 16 * kUnits ? ks + at / DP * kKStride + at % DP
                                      : vs + vat / kKv8Page * kVStride + vat % kKv8Page;
      *reinterpret_cast<v8h *>(to) = kv8_halves(code[u][0], code[u][1]);
      *reinterpret_cast<v8h *>(to + 8) = kv8_halves(code[u][2], code[u][3]);
    }
    const float pf = f, plg = lg, piv = iv;
    __syncthreads();
    if (p + 1 < span.p1) fetch(p + 1);

    const int token = p * kKv8Page;
    v16f x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
      const int at = 32 * t + 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const v8h k = *reinterpret_cast<const v8h *>(ks + at * kKStride + 16 * st + 8 * half);
        x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[st], x[t], 0, 0, 0);
      }
    }
    const bool cut = token < all_lo || token + kKv8Page - 1 > all_hi;
    float most = kNegInf;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float v = __builtin_fmaf(x[t][i], pf, plg);
        const int key = token + 32 * t + 16 * (i >> 3) + 8 * half + (i & 7);
        if (cut && (key < key_lo || key > key_hi)) v = kNegInf;
        x[t][i] = v;
        most = fmaxf(most, v);
      }
    most = max_xor32(most);
    if (__any(most > m + kMost)) {
      const float now = most > m + kMost ? most - kSet : m;
      const float keep = m == now ? 1.f : exp2_fast(m - now);
      m = now;
      l *= keep;
#pragma unroll
      for (int t = 0; t < kOut; ++t) o[t] *= keep;
    }
    const float ref = m == kNegInf ? 0.f : m;  // no key yet
    float sum = 0.f;
    v8h w[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = exp2_fast(x[t][i] - ref);
        sum += e;
        w[2 * t + (i >> 3)][i & 7] = (_Float16)e;
      }
    l = __builtin_fmaf(sum, piv, l);
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const v8h v = *reinterpret_cast<const v8h *>(vs + (32 * t + col) * kVStride + 16 * j + 8 * half);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, w[j], o[t], 0, 0, 0);
      }
  }

  l += __shfl_xor(l, 32);
  if (!in) return;
  // a row that sees no key: as its position says, not as its sum does
  const bool empty = len == 0 || (a.causal && pos < 0);
  const float scale = 1.f / l;
  const int64_t at = (int64_t)(rows.row0 + qi) * a.Hq + head;
#pragma unroll
  for (int t = 0; t < kOut; ++t)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * t + 2 * i + 4 * half;
      if (d >= a.D) continue;
      v2u y;
      y[0] = __builtin_bit_cast(uint32_t, pack_half(o[t][i] * scale, o[t][i + 1] * scale));
      y[1] = __builtin_bit_cast(uint32_t, pack_half(o[t][i + 2] * scale, o[t][i + 3] * scale));
      if (empty) y = v2u{0u, 0u};
      *reinterpret_cast<v2u *>(a.Y + at * a.D + d) = y;
    }
  if (half == 0 && a.lse != nullptr) a.lse[at] = empty ? kNegInf : (m + log2f(l)) * kLn2;
}

}  // namespace detail

hipError_t launch_kv8_tiles(const Kv8Attn &a, hipStream_t st) {
  const int64_t slots = kv8_tile_slots((int64_t)a.T * (a.Hq / a.Hkv), a.B, detail::kTileRows);
  const unsigned grid = (unsigned)(slots * a.Hkv);
  switch (kv8_width(a.D)) {
    case 64: detail::kv8_tile_kernel<64><<<grid, 256, 0, st>>>(a); break;
    case 96: detail::kv8_tile_kernel<96><<<grid, 256, 0, st>>>(a); break;
    case 128: detail::kv8_tile_kernel<128><<<grid, 256, 0, st>>>(a); break;
    case 192: detail::kv8_tile_kernel<192><<<grid, 256, 0, st>>>(a); break;
    default: detail::kv8_tile_kernel<256><<<grid, 256, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace ot
