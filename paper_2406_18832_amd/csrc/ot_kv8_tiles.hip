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

template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP > 192 ? 1 : 2) void kv8_tile_kernel(Kv8Attn a) {
  constexpr int kThreads = 64 * WAVES, kRows = 32 * WAVES;
  constexpr int kKStride = DP + 8, kVStride = kKv8Page + 8;  // halves; off the banks
  constexpr int kSteps = DP / 16, kOut = DP / 32;
  constexpr int kUnits = DP * kKv8Page / 16;     // 16 bytes each, of K as of V
  constexpr int kLoads = (2 * kUnits + kThreads - 1) / kThreads;  // K's units, then V's
  static_assert(kUnits % 64 == 0, "whole waves");
  __shared__ __attribute__((aligned(16))) _Float16 ks[2][kKv8Page * kKStride];
  __shared__ __attribute__((aligned(16))) _Float16 vs[2][DP * kVStride];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int h = blockIdx.x % a.Hkv;
  const int64_t slot = blockIdx.x / a.Hkv;
  const int G = a.Hq / a.Hkv;
  const int b = kv8_find(a.B, lane, slot,
                         [&](int i) { return kv8_tile_slot((int64_t)a.cu[i] * G, i, kRows); });
  if (b < 0) return;
  const Kv8Rows rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
  // counted from the end: under a causal mask the last tile has the most pages
  const int64_t tiles = ((int64_t)rows.n * G + kRows - 1) / kRows;
  const int64_t tile = tiles - 1 - (slot - kv8_tile_slot((int64_t)a.cu[b] * G, b, kRows));
  if (tile < 0 || tile >= tiles) return;
  const int64_t len0 = a.kv_len[b];
  const int len = (int)kv8_len(len0, a.cache.max_pages);
  const bool bad = len0 > len;
  const int row0 = (int)tile * kRows + 32 * wave;
  const int all = rows.n * G;
  const int first = (int)tile * kRows / G;
  const int last = min((int)(tile + 1) * kRows - 1, all - 1) / G;
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
    if (a.scale < 0.f) w ^= 0x80008000u;  // the factor of a score is not negative then
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
  const float fac = fabsf(a.scale) * kLog2e;

  v4u code[kLoads];
  float f = 0.f, lg = 0.f, iv = 1.f;
  // page p's codes on their way into registers, and its scales
  auto fetch = [&](int p) {
    int64_t page = kv8_page(a.cache.table, b, p, a.cache.max_pages, a.cache.num_pages);
    const bool none = page < 0 || bad;
    if (page < 0) page = 0;
    const int64_t ph = page * a.Hkv + h;
    const __amdgpu_buffer_rsrc_t keys = make_rsrc(a.cache.Kc + ph * (DP * kKv8Page), DP * kKv8Page);
    const __amdgpu_buffer_rsrc_t values = make_rsrc(a.cache.Vc + ph * (DP * kKv8Page), DP * kKv8Page);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * kThreads + wave * 64;  // a wave's are all of one kind
      if (at < kUnits)
        code[u] = __builtin_amdgcn_raw_buffer_load_b128(keys, (u * kThreads + tid) * 16, 0, 0);
      else if (at < 2 * kUnits)
        code[u] = __builtin_amdgcn_raw_buffer_load_b128(values, (u * kThreads + tid - kUnits) * 16, 0, 0);
    }
    f = none ? __builtin_nanf("") : a.cache.Ks[ph] * fac;
    value_scale(none ? 0.f : a.cache.Vs[ph], lg, iv);
  };
  // and as fp16 into LDS
  auto stage = [&](int to) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (u * kThreads + wave * 64 >= 2 * kUnits) break;
      const int at = (u * kThreads + tid) * 16, vat = at - 16 * kUnits;
      _Float16 *p = u * kThreads + wave * 64 < kUnits
                        ? ks[to] + at / DP * kKStride + at % DP
                        : vs[to] + vat / kKv8Page * kVStride + vat % kKv8Page;
      *reinterpret_cast<v8h *>(p) = kv8_halves(code[u][0], code[u][1]);
      *reinterpret_cast<v8h *>(p + 8) = kv8_halves(code[u][2], code[u][3]);
    }
  };
  const int key_row = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
  if (span.p0 < span.p1) {
    fetch(span.p0);
    stage(0);
  }
  for (int p = span.p0, buf = 0; p < span.p1; ++p, buf ^= 1) {
    const float pf = f, plg = lg, piv = iv;
    __syncthreads();  // this page is there, and the one before is done with
    const bool more = p + 1 < span.p1;
    if (more) fetch(p + 1);
    const _Float16 *kp = ks[buf] + key_row * kKStride + 8 * half;
    const _Float16 *vp = vs[buf] + col * kVStride + 8 * half;

    const int token = p * kKv8Page;
    v16f x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const v8h k = *reinterpret_cast<const v8h *>(kp + 32 * t * kKStride + 16 * st);
        x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[st], x[t], 0, 0, 0);
      }
    }
    const bool cut = token < all_lo || token + kKv8Page - 1 > all_hi;
    auto hidden = [&](int t, int i) {
      const int key = token + 32 * t + 16 * (i >> 3) + 8 * half + (i & 7);
      return key < key_lo || key > key_hi;
    };
    if (cut) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (hidden(t, i)) x[t][i] = kNegInf;
    }
    float most = kNegInf;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, x[t][i]);
    most = __builtin_fmaf(max_xor32(most), pf, plg);  // pf >= 0: a row's largest exponent
    if (__any(most > m + kMost)) {
      const float now = most > m + kMost ? most - kSet : m;
      const float keep = m == now ? 1.f : exp2_fast(m - now);
      m = now;
      l *= keep;
#pragma unroll
      for (int t = 0; t < kOut; ++t) o[t] *= keep;
    }
    const float off = plg - (m == kNegInf ? 0.f : m);  // no key yet
    float sum = 0.f;
    v8h w[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = __builtin_fmaf(x[t][i], pf, off);
    if (cut) {  // a scale of 0 has made NaN of them
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (hidden(t, i)) x[t][i] = kNegInf;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = exp2_fast(x[t][i]);
        sum += e;
        w[2 * t + (i >> 3)][i & 7] = (_Float16)e;
      }
    l = __builtin_fmaf(sum, piv, l);
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const v8h v = *reinterpret_cast<const v8h *>(vp + 32 * t * kVStride + 16 * j);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, w[j], o[t], 0, 0, 0);
      }
    if (more) stage(buf ^ 1);
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

template <int DP, int WAVES>
static hipError_t tile_launch(const Kv8Attn &a, hipStream_t st) {
  const int64_t slots = kv8_tile_slots((int64_t)a.T * (a.Hq / a.Hkv), a.B, 32 * WAVES);
  detail::kv8_tile_kernel<DP, WAVES><<<(unsigned)(slots * a.Hkv), 64 * WAVES, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv8_tiles(const Kv8Attn &a, hipStream_t st) {
  switch (kv8_width(a.D)) {
    case 64: return tile_launch<64, 8>(a, st);
    case 96: return tile_launch<96, 8>(a, st);
    case 128: return tile_launch<128, 8>(a, st);
    case 192: return tile_launch<192, 8>(a, st);
    default: return tile_launch<256, 4>(a, st);
  }
}

}  // namespace ot
