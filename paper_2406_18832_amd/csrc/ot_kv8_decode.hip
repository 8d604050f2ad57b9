// Attention over the 8-bit cache for few query rows: decode, and drafts of a few
// tokens.  It reads every code once and is bound by that.
//
// A workgroup takes one key head and a run of a sequence's pages; its four waves
// take the pages in turn, each with a running maximum, sum and output of its own
// (no barrier until they meet at the end).  Up to 16 query rows (tokens times the
// query heads of the key head) are the 16 columns of v_mfma_f32_16x16x32_f16, 32
// those of two; with a single row 15/16 of the matrix cores' work is for nothing,
// which costs less than the loads take.
//
// MI355X, cache bytes per time, where a large read reaches 6.2 TB/s: 4 sequences of
// 32000-131000 keys of 8 heads of 128 channels with 4 query heads each 109 us (6.1 TB/s),
// 64 sequences of 100-2047 keys of 40 heads 127 us (5.6), 5 tokens of 16 sequences of
// 900-8000 keys 37 us (4.0: four or five pages to a wave, and the joining).  One sequence
// of 200 keys is 5 us, three memory latencies behind each other.  Codes pass the caches
// by (with them kept 147 us in place of 130), and the card is filled once: with more and
// smaller items their starts and their joining cost more than the evener end gives.
//
// Lane l has query row l mod 16 and, with g = l / 16, tokens 16 g .. 16 g + 15 of a
// page: K's row 4 g' + i of the s-th of four products is token 16 g' + 4 s + i.
// V^T's rows are channels, its 16 bytes of a lane are tokens 16 g .. of one channel.
#include <math.h>

#include <type_traits>

#include "ot_kv8_attn.h"

namespace ot {
namespace detail {

constexpr int kDecodeWaves = 4;
// In how many parts the waves' outputs meet: some 8 tiles of 16 channels and rows at a time.
constexpr int kv8_meetings(int out, int tiles) {
  int n = (out * tiles + 7) / 8;
  while (out % n != 0) --n;
  return n;
}
constexpr int kNonTemporal = 2;  // buffer load hint: codes are read once

// The first DC channels of DP.
template <int DP, int DC, int RT>
__global__ __launch_bounds__(64 * kDecodeWaves, kv8_decode_waves(DP, RT)) void kv8_decode_kernel(Kv8Attn a, Kv8Split s) {
  constexpr int kSteps = (DC + 31) / 32, kOut = DC / 16;
  constexpr int kChunks = kSteps / 2, kTail = kSteps % 2;  // of a key's row
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int h = blockIdx.y;
  const int G = a.Hq / a.Hkv;

  // Where a workgroup does not take 32 rows, an item's two row tiles are eight workgroups
  // apart, and read its pages through one L2 (30 sequences of 1000-20000 keys of 2 x 24 heads
  // of 256 channels 109 us, one after the other 124).
  int z = 0, number = blockIdx.x;
  if (kv8_decode_tiles(DP, 32) == 1 && a.max_q * G > 16) {
    z = blockIdx.x / 8 % 2;
    number = blockIdx.x / 16 * 8 + blockIdx.x % 8;
  }
  const Kv8Item item = kv8_item(a, lane, number, s.wanted, s.least);
  if (item.b < 0) return;
  const Kv8Seq seq = kv8_seq(a, item.b);
  const int rows = min(seq.rows.n, a.max_q) * G, row_base = z * (16 * RT);
  if (z == 0 && h == 0 && item.index == 0 && threadIdx.x == 0 && s.wanted != 0)
    s.spans[item.b] = make_int2(item.first, item.count);
  if (row_base >= rows) return;
  const int p0 = seq.span.p0 + item.index * item.chunk;
  const int p1 = p0 + min(item.chunk, seq.span.p1 - p0);

  // this lane's query rows, and the positions of the keys that they see
  v8h q[RT][kSteps];
  int key_lo[RT], key_hi[RT];  // [lo, hi]
  int all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row_base + 16 * r + col;
    const bool in = row < rows;
    const int i = in ? row / G : 0;
    const uint16_t *p = a.q + (seq.rows.row0 + i) * a.ldq + (h * G + (in ? row % G : 0)) * a.D;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const int d = st < 2 * kChunks ? 64 * (st >> 1) + 16 * g + 8 * (st & 1) : 64 * kChunks + 8 * g;
      v4u w = {0u, 0u, 0u, 0u};
      if (in && d < a.D) w = *reinterpret_cast<const v4u *>(p + d);
      q[r][st] = __builtin_bit_cast(v8h, w);
    }
    const int pos = (int)(seq.len - seq.rows.n + i);
    key_hi[r] = a.causal ? pos : (int)seq.len - 1;
    key_lo[r] = a.window > 0 ? (int)kv8_max(0, pos - a.window + 1) : 0;
  }
  // keys that every row sees: those after the last row's first and up to the first
  // row's last
  if (a.causal) all_hi = (int)(seq.len - seq.rows.n);
  all_hi = min(all_hi, (int)seq.len - 1);
  if (a.window > 0) all_lo = (int)kv8_max(0, seq.len - a.window);

  float m[RT], l[RT];
  v4f o[RT][kOut];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = kNegInf;
    l[r] = 0.f;
#pragma unroll
    for (int t = 0; t < kOut; ++t) o[r][t] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  const float fac = a.scale * kLog2e;
  const int key_at = (16 * (col >> 2) + (col & 3)) * DP + 16 * g, value_at = col * kKv8Page + 16 * g;

  // 64 of this wave's pages at a time: lane i has the i-th one's number and scales.  A
  // page's keys are fetched while the one before goes through softmax and values, its
  // values from there until its own scores are there: both take the registers that the
  // page before has just left.
  for (int batch = p0 + wave; batch < p1; batch += 64 * kDecodeWaves) {
    const int mine = batch + kDecodeWaves * lane;
    const int todo = min(64, (p1 - batch + kDecodeWaves - 1) / kDecodeWaves);
    int64_t page = -1;
    if (mine < p1)
      page = kv8_page(a.cache.table, item.b, mine, a.cache.max_pages, a.cache.num_pages);
    const bool none = page < 0;
    const int at = none ? 0 : (int)page;  // its scale is NaN: what sees it is
    v4u kc[4][kChunks > 0 ? kChunks : 1];
    v2u kt[4];
    v4u vc[kOut];
    auto load_keys = [&](int n) {
      const int64_t ph = (int64_t)__builtin_amdgcn_readlane(at, n) * a.Hkv + h;
      const __amdgpu_buffer_rsrc_t keys = make_rsrc(a.cache.Kc + ph * (DP * kKv8Page), DP * kKv8Page);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
          kc[t][c] = __builtin_amdgcn_raw_buffer_load_b128(keys, key_at, 4 * t * DP + 64 * c, kNonTemporal);
        if constexpr (kTail != 0)
          kt[t] = __builtin_amdgcn_raw_buffer_load_b64(keys, key_at - 8 * g, 4 * t * DP + 64 * kChunks, kNonTemporal);
      }
    };
    auto load_values = [&](int n) {
      const int64_t ph = (int64_t)__builtin_amdgcn_readlane(at, n) * a.Hkv + h;
      const __amdgpu_buffer_rsrc_t values = make_rsrc(a.cache.Vc + ph * (DP * kKv8Page), DP * kKv8Page);
#pragma unroll
      for (int t = 0; t < kOut; ++t)
        vc[t] = __builtin_amdgcn_raw_buffer_load_b128(values, value_at, 1024 * t, kNonTemporal);
    };
    float ks = __builtin_nanf(""), vs = 0.f;
    if (!none) {
      ks = a.cache.Ks[page * a.Hkv + h];
      vs = a.cache.Vs[page * a.Hkv + h];
    }
    load_keys(0);
    load_values(0);
    float lg, inv;
    value_scale(vs, lg, inv);
    ks = seq.bad ? __builtin_nanf("") : ks * fac;

    // keeps the scheduler from fetching into fresh registers, which there are none of
    auto phase = [] { __builtin_amdgcn_sched_barrier(0); };
    auto one_page = [&](int n, auto more) {
      const float f = lane_float(ks, n), lgv = lane_float(lg, n), iv = lane_float(inv, n);
      v4f x[RT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int r = 0; r < RT; ++r) x[r][t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          v8h k;
          if (st < 2 * kChunks) {
            const v4u w = kc[t][st >> 1];
            k = (st & 1) ? kv8_halves(w[2], w[3]) : kv8_halves(w[0], w[1]);
          } else {
            k = kv8_halves(kt[t][0], kt[t][1]);
          }
#pragma unroll
          for (int r = 0; r < RT; ++r)
            x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[r][st], x[r][t], 0, 0, 0);
        }
        if (DP * RT >= 128) phase();
      }
      phase();
      if constexpr (more) load_keys(n + 1);
      phase();
      const int token = (batch + kDecodeWaves * n) * kKv8Page;
      const bool cut = token < all_lo || token + kKv8Page - 1 > all_hi;
      v8h p[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float most = kNegInf;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[r][t][i] = __builtin_fmaf(x[r][t][i], f, lgv);
        }
        if (cut) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = token + 16 * g + 4 * t + i;
              if (key < key_lo[r] || key > key_hi[r]) x[r][t][i] = kNegInf;
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = fmaxf(most, x[r][t][i]);
        most = max_xor32(max_xor16(most));
        if (__any(most - m[r] > kMost)) {
          const float now = most - m[r] > kMost ? raise_ref(m[r], most) : m[r];
          const float keep = m[r] == now ? 1.f : exp2_fast(m[r] - now);
          m[r] = now;
          l[r] *= keep;
#pragma unroll
          for (int t = 0; t < kOut; ++t) o[r][t] *= keep;
        }
        const float ref = m[r] == kNegInf ? 0.f : m[r];  // no key yet
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = exp2_fast(x[r][t][i] - ref);
            sum += w[i];
          }
          const v2h lo = pack_half(w[0], w[1]), hi = pack_half(w[2], w[3]);
          p[r][t >> 1][4 * (t & 1) + 0] = lo[0];
          p[r][t >> 1][4 * (t & 1) + 1] = lo[1];
          p[r][t >> 1][4 * (t & 1) + 2] = hi[0];
          p[r][t >> 1][4 * (t & 1) + 3] = hi[1];
        }
        l[r] = __builtin_fmaf(sum, iv, l[r]);
      }
      phase();
#pragma unroll
      for (int t = 0; t < kOut; ++t) {
        const v8h v0 = kv8_halves(vc[t][0], vc[t][1]), v1 = kv8_halves(vc[t][2], vc[t][3]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[r][0], o[r][t], 0, 0, 0);
          o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[r][1], o[r][t], 0, 0, 0);
        }
        if (DP * RT >= 128 && t % 2 == 1) phase();
      }
      phase();
      if constexpr (more) load_values(n + 1);
      phase();
    };
    for (int n = 0; n + 1 < todo; ++n) one_page(n, std::true_type{});
    one_page(todo - 1, std::false_type{});
  }

  // The waves' results meet, some channels at a time; only rows that exist are written.
  constexpr int kRows = 16 * RT;
  constexpr int kGroups = kv8_meetings(kOut, RT), kPer = kOut / kGroups, kCols = 16 * kPer;
  static_assert(kPer * kGroups == kOut, "whole groups");
  __shared__ float meet_m[kDecodeWaves][kRows], meet_l[kDecodeWaves][kRows];
  __shared__ __attribute__((aligned(16))) float meet_o[kDecodeWaves][kRows][kCols];
  const int here = min(rows - row_base, kRows);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (g == 0) {
      meet_m[wave][16 * r + col] = m[r];
      meet_l[wave][16 * r + col] = l[r];
    }
  }
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    if (u > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
      if (16 * r + col < here) {
#pragma unroll
        for (int t = 0; t < kPer; ++t)
          *reinterpret_cast<v4f *>(&meet_o[wave][16 * r + col][16 * t + 4 * g]) = o[r][u * kPer + t];
      }
    __syncthreads();
    for (int e = threadIdx.x; e < here * (kCols / 4); e += 64 * kDecodeWaves) {
      const int row = e / (kCols / 4), c = e % (kCols / 4) * 4, d = u * kCols + c;
      float top = kNegInf;
#pragma unroll
      for (int w = 0; w < kDecodeWaves; ++w) top = fmaxf(top, meet_m[w][row]);
      const float ref = top == kNegInf ? 0.f : top;
      float sum = 0.f;
      v4f out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kDecodeWaves; ++w) {
        const float part = exp2_fast(meet_m[w][row] - ref);
        sum = __builtin_fmaf(part, meet_l[w][row], sum);
        const v4f v = *reinterpret_cast<const v4f *>(&meet_o[w][row][c]);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = __builtin_fmaf(part, v[i], out[i]);
      }
      const int full = row_base + row;
      if (item.count == 1) {
        const int i = full / G, head = h * G + full % G;
        const int64_t pos = seq.len - seq.rows.n + i;
        // a row that sees no key: as its position says, not as its sum does
        const bool empty = kv8_empty(a, seq.len, pos, seq.bad);
        if (seq.bad) sum = __builtin_nanf("");
        const int64_t at = (int64_t)(seq.rows.row0 + i) * a.Hq + head;
        const float scale = 1.f / sum;
        if (d < a.D) {
          v2u y;
          y[0] = __builtin_bit_cast(uint32_t, pack_half(out[0] * scale, out[1] * scale));
          y[1] = __builtin_bit_cast(uint32_t, pack_half(out[2] * scale, out[3] * scale));
          if (empty) y = v2u{0u, 0u};
          *reinterpret_cast<v2u *>(a.Y + at * a.D + d) = y;
        }
        if (d == 0 && a.lse != nullptr)
          a.lse[at] = empty ? kNegInf : (top + log2f(sum)) * kLn2;
      } else {
        const int64_t at = kv8_partial(number, h, full, a.Hkv, s.rows);
        if (d == 0) {
          s.m[at] = top;
          s.l[at] = sum;
        }
        *reinterpret_cast<v4f *>(s.o + at * DP + d) = out;
      }
    }
  }
}

// The items of a sequence joined: a wave to a query row of a key head at a time, or four
// (`team`) where there are many items, which they take in turn, eight items' loads at a
// time.
template <int DP>
__global__ __launch_bounds__(256) void kv8_combine_kernel(Kv8Attn a, Kv8Split s) {
  constexpr int kPer = (DP + 63) / 64, kAhead = 8;
  __shared__ float meet[4][2 + 64 * kPer];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = blockIdx.y, G = a.Hq / a.Hkv;
  const Kv8Rows rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
  if (rows.n == 0) return;
  const int2 span = s.spans[b];
  if (span.y <= 1) return;
  const int64_t whole = a.kv_len[b], len = kv8_len(whole, a.cache.max_pages);
  const bool bad = whole > len;
  const int mine = min(rows.n, a.max_q) * G, all = a.Hkv * mine;
  const int team = span.y > 2 * kAhead ? 4 : 1, first = team == 4 ? wave : 0;
  for (int base = blockIdx.x * (4 / team); base < all; base += gridDim.x * (4 / team)) {
    const int which = team == 4 ? base : min(base + wave, all - 1);
    const int h = which / mine, row = which % mine;
    const int64_t from = kv8_partial(span.x, h, row, a.Hkv, s.rows), step = a.Hkv * s.rows;
    float top = kNegInf, sum = 0.f, out[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) out[i] = 0.f;
    for (int c0 = first * kAhead; c0 < span.y; c0 += team * kAhead) {
      float m[kAhead], l[kAhead], v[kAhead][kPer];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const bool in = c0 + j < span.y;
        const int64_t at = from + (in ? c0 + j : c0) * step;
        m[j] = in ? s.m[at] : kNegInf;
        l[j] = in ? s.l[at] : 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int d = 64 * i + lane;
          v[j][i] = in && (DP % 64 == 0 || d < DP) ? s.o[at * DP + d] : 0.f;
        }
      }
      float now = top;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) now = fmaxf(now, m[j]);
      const float ref = now == kNegInf ? 0.f : now, keep = exp2_fast(top - ref);
      top = now;
      sum *= keep;
#pragma unroll
      for (int i = 0; i < kPer; ++i) out[i] *= keep;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const float part = exp2_fast(m[j] - ref);
        sum = __builtin_fmaf(part, l[j], sum);
#pragma unroll
        for (int i = 0; i < kPer; ++i) out[i] = __builtin_fmaf(part, v[j][i], out[i]);
      }
    }
    if (team == 4) {
      __syncthreads();  // the row before is done with
      if (lane == 0) {
        meet[wave][0] = top;
        meet[wave][1] = sum;
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) meet[wave][2 + 64 * i + lane] = out[i];
      __syncthreads();
      if (wave != 0) continue;
      top = fmaxf(fmaxf(meet[0][0], meet[1][0]), fmaxf(meet[2][0], meet[3][0]));
      const float ref = top == kNegInf ? 0.f : top;
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) out[i] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float part = exp2_fast(meet[w][0] - ref);
        sum = __builtin_fmaf(part, meet[w][1], sum);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          out[i] = __builtin_fmaf(part, meet[w][2 + 64 * i + lane], out[i]);
      }
    } else if (base + wave >= all) {
      continue;
    }
    const int i = row / G, head = h * G + row % G;
    const bool empty = kv8_empty(a, len, len - rows.n + i, bad);
    if (bad) sum = __builtin_nanf("");
    const int64_t at = (int64_t)(rows.row0 + i) * a.Hq + head;
    const float scale = 1.f / sum;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (64 * j + lane < a.D)
        a.Y[at * a.D + 64 * j + lane] = empty ? 0 : float_to_half_bits(out[j] * scale);
    if (lane == 0 && a.lse != nullptr) a.lse[at] = empty ? kNegInf : (top + log2f(sum)) * kLn2;
  }
}

// The parts of tiles' rows joined: a wave to a row of a head, four parts' loads at a time.
template <int DP>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8Attn a, Kv8Parts p) {
  constexpr int kPer = (DP + 63) / 64, kAhead = 4;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  // rows of no sequence have no count
  if (row >= p.rows || row < (int64_t)a.cu[0] * a.Hq || row >= (int64_t)a.cu[a.B] * a.Hq) return;
  const int marked = p.counts[row];  // below 0: the row sees no key
  const int count = min(abs(marked), p.parts);
  if (count <= 1) return;
  float top = kNegInf, sum = 0.f, out[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) out[i] = 0.f;
  for (int c0 = 0; c0 < count; c0 += kAhead) {
    float m[kAhead], l[kAhead], v[kAhead][kPer];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const bool in = c0 + j < count;
      const int64_t at = (in ? c0 + j : c0) * p.rows + row;
      m[j] = in ? p.m[at] : kNegInf;
      l[j] = in ? p.l[at] : 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int d = 64 * i + lane;
        v[j][i] = in && (DP % 64 == 0 || d < DP) ? p.o[at * DP + d] : 0.f;
      }
    }
    float now = top;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) now = fmaxf(now, m[j]);
    const float ref = now == kNegInf ? 0.f : now, keep = exp2_fast(top - ref);
    top = now;
    sum *= keep;
#pragma unroll
    for (int i = 0; i < kPer; ++i) out[i] *= keep;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const float part = exp2_fast(m[j] - ref);
      sum = __builtin_fmaf(part, l[j], sum);
#pragma unroll
      for (int i = 0; i < kPer; ++i) out[i] = __builtin_fmaf(part, v[j][i], out[i]);
    }
  }
  const float scale = 1.f / sum;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (64 * j + lane < a.D)
      a.Y[row * a.D + 64 * j + lane] = marked < 0 ? 0 : float_to_half_bits(out[j] * scale);
  if (lane == 0 && a.lse != nullptr)
    a.lse[row] = marked < 0 ? kNegInf : (top + log2f(sum)) * kLn2;
}

template <int DP, int DC, int RT>
hipError_t decode_launch(const Kv8Attn &a, int64_t max_rows, const Kv8Split &s, hipStream_t st) {
  static_assert(kFewRows <= 32, "two row tiles at most");
  const bool two = max_rows > 16 * RT;
  const dim3 grid((unsigned)(two ? (s.items + 7) / 8 * 16 : s.items), (unsigned)a.Hkv);
  kv8_decode_kernel<DP, DC, RT><<<grid, 64 * kDecodeWaves, 0, st>>>(a, s);
  return hipGetLastError();
}

template <int DP, int DC = DP>
hipError_t decode_width(const Kv8Attn &a, int64_t max_rows, const Kv8Split &s, hipStream_t st) {
  if constexpr (kv8_decode_tiles(DP, 32) == 2)
    if (max_rows > 16) return decode_launch<DP, DC, 2>(a, max_rows, s, st);
  return decode_launch<DP, DC, 1>(a, max_rows, s, st);
}

}  // namespace detail

hipError_t launch_kv8_decode(const Kv8Attn &a, const Kv8Split &s, hipStream_t st) {
  const int64_t max_rows = (int64_t)a.max_q * (a.Hq / a.Hkv);
  // The widths that a head's 16 channels make, but for the narrowest and the widest, whose
  // time is a whole page's: 16 sequences of 8000 keys of 8 heads 89 us with 208 as with 256
  // channels, 32 of 16 heads 95 with 16 as with 64.
  switch ((a.D + 15) / 16) {
    case 5: return detail::decode_width<96, 80>(a, max_rows, s, st);
    case 6: return detail::decode_width<96>(a, max_rows, s, st);
    case 7: return detail::decode_width<128, 112>(a, max_rows, s, st);
    case 8: return detail::decode_width<128>(a, max_rows, s, st);
    case 9: return detail::decode_width<192, 144>(a, max_rows, s, st);
    case 10: return detail::decode_width<192, 160>(a, max_rows, s, st);
    case 11: return detail::decode_width<192, 176>(a, max_rows, s, st);
    case 12: return detail::decode_width<192>(a, max_rows, s, st);
    default:
      return a.D <= 64 ? detail::decode_width<64>(a, max_rows, s, st)
                       : detail::decode_width<256>(a, max_rows, s, st);
  }
}

hipError_t launch_kv8_combine(const Kv8Attn &a, const Kv8Split &s, hipStream_t st) {
  // a row to a wave; more workgroups where there are few sequences, which may have many
  // items each
  const int64_t rows = s.rows * a.Hkv, share = kv8_max((rows + 3) / 4, 512 / a.B);
  const dim3 grid((unsigned)kv8_min(rows, share), (unsigned)a.B);
  switch (kv8_width(a.D)) {
    case 64: detail::kv8_combine_kernel<64><<<grid, 256, 0, st>>>(a, s); break;
    case 96: detail::kv8_combine_kernel<96><<<grid, 256, 0, st>>>(a, s); break;
    case 128: detail::kv8_combine_kernel<128><<<grid, 256, 0, st>>>(a, s); break;
    case 192: detail::kv8_combine_kernel<192><<<grid, 256, 0, st>>>(a, s); break;
    default: detail::kv8_combine_kernel<256><<<grid, 256, 0, st>>>(a, s); break;
  }
  return hipGetLastError();
}

hipError_t launch_kv8_join(const Kv8Attn &a, const Kv8Parts &p, hipStream_t st) {
  const unsigned grid = (unsigned)((p.rows + 3) / 4);
  switch (kv8_width(a.D)) {
    case 64: detail::kv8_join_kernel<64><<<grid, 256, 0, st>>>(a, p); break;
    case 96: detail::kv8_join_kernel<96><<<grid, 256, 0, st>>>(a, p); break;
    case 128: detail::kv8_join_kernel<128><<<grid, 256, 0, st>>>(a, p); break;
    case 192: detail::kv8_join_kernel<192><<<grid, 256, 0, st>>>(a, p); break;
    default: detail::kv8_join_kernel<256><<<grid, 256, 0, st>>>(a, p); break;
  }
  return hipGetLastError();
}

}  // namespace ot
