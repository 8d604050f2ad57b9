// Attention over the 8-bit cache for many query rows (prompts, pieces of prompts): bound
// by the matrix cores and the vector instructions beside them.  A wave's products of a
// page of 128 channels take 1024 cycles, as long as LDS takes for their A operands, and
// its other work (the softmax of 2048 scores, its share of the codes) some 240 vector
// instructions, of which five or six find a place beside each product.
//
// MI355X, of 1276 TFLOP/s that a large fp16 library product reaches: an 8192-token prompt
// of 72 heads 1165-1270 us (1060-975 TFLOP/s of what the mask leaves; cards differ by their
// clocks under load); 4096-8192 tokens of 32 heads without a mask 1130 TFLOP/s at 128 channels, 1190 at 192, 920 at 96, 770 at 64
// (fewer products to a score) and 770 at 256 (registers for one wave to a SIMD).
//
// A workgroup takes a tile of query rows (tokens times the query heads of one key head)
// of a sequence, 32 to each of its waves, and goes over the pages that they see.  A
// page's codes are turned to fp16 once, on their way into LDS, where all waves read them
// as the A operands of v_mfma_f32_32x32x16_f16.
//
// S^T = K Q^T: lane l has query row l mod 32; K's row 8 a + 4 h + i of a tile of 32
// tokens is token 16 (a / 2) + 8 h + 4 (a mod 2) + i, so that the 16 results of a lane
// (h = l / 32; a, i) are the weights of two runs of eight tokens, each the lane's part
// of the B operand of one product O^T += V^T P^T.
#include <math.h>

#include <type_traits>

#include "ot_kv8_attn.h"

namespace ot {
namespace detail {

// A sequence's tiles, and the pages of its first and its last one.
struct Kv8Tiles {
  Kv8Rows rows;
  int kv_len, tiles, first, last;
};
template <int kRows>
__device__ __forceinline__ Kv8Tiles kv8_tiles(const Kv8Attn &a, int b) {
  Kv8Tiles s{{0, 0}, 0, 0, 0, 0};
  if (b >= a.B) return s;
  s.rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
  s.kv_len = a.kv_len[b];
  const int G = a.Hq / a.Hkv, n = s.rows.n;
  s.tiles = (int)(((int64_t)n * G + kRows - 1) / kRows);
  const int64_t len = kv8_len(s.kv_len, a.cache.max_pages), q = kv8_min((kRows + G - 1) / G, n);
  const Kv8Span first = kv8_span(len, n, 0, q, a.causal, a.window);
  const Kv8Span last = kv8_span(len, n, n - q, q, a.causal, a.window);
  s.first = first.p1 - first.p0;
  s.last = last.p1 - last.p0;
  return s;
}

// Which tile a key head's i-th workgroup takes, and which part of its pages.
struct Kv8Slot {
  int b;  // sequence, or -1
  int64_t tile;
  int part, parts, most;  // of at most so many with so many pages each
  Kv8Rows rows;           // the sequence's, and its keys
  int kv_len;
};

// With tiles' pages shared between workgroups: all of a sequence's tiles come in as many
// parts as its last one needs.  A part has a quarter over a workgroup's even share of all
// pages (those of a sequence's tiles taken to lie evenly between the first one's and the
// last one's), or more where the launch has too few workgroups for that.
template <int kRows>
__device__ __forceinline__ Kv8Slot kv8_part(const Kv8Attn &a, const Kv8Parts &p, int i, int lane) {
  const Kv8Tiles front = kv8_tiles<kRows>(a, lane);
  const auto seq = [&](int b0) { return b0 == 0 ? front : kv8_tiles<kRows>(a, b0 + lane); };
  float pages = 0.f;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const Kv8Tiles s = seq(b0);
    pages += 0.5f * (float)s.tiles * (float)(s.first + s.last);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) pages += __shfl_xor(pages, off);
  int most = max(p.least, (int)fminf(1.25f * pages * (float)a.Hkv / (float)p.groups, 1e9f) + 1);
  const auto parts = [&](const Kv8Tiles &s) { return max(min((s.last + most - 1) / most, p.parts), 1); };
  for (;; most += most / 4 + 1) {
    int all = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      const Kv8Tiles s = seq(b0);
      all += s.tiles * parts(s);
    }
    if (__builtin_amdgcn_readlane(wave_upto(all), 63) <= p.slots || most > a.cache.max_pages) break;
  }
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const Kv8Tiles s = seq(b0);
    const int own = s.tiles * parts(s), upto = wave_upto(own);
    const uint64_t past = __ballot(before + upto > i);
    if (past != 0) {
      const int at = __builtin_ctzll(past), count = __builtin_amdgcn_readlane(parts(s), at);
      const int j = i - before - __builtin_amdgcn_readlane(upto - own, at);
      return {b0 + at, __builtin_amdgcn_readlane(s.tiles, at) - 1 - j / count, j % count, count, most,
              {__builtin_amdgcn_readlane(s.rows.row0, at), __builtin_amdgcn_readlane(s.rows.n, at)},
              __builtin_amdgcn_readlane(s.kv_len, at)};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0, 0, {0, 0}, 0};
}

// A workgroup to a tile.  A few sequences' tiles come in the order of their pages, the
// most first (under a causal mask a tile's pages go with its number, and its sequence's
// earlier tokens count as tiles in front of it), so that the last ones to run are short:
// with S(x) the number of tiles with x and more tiles before them, the i-th tile is among
// those with the largest x that S(x) > i has.
template <int kRows>
__device__ __forceinline__ Kv8Slot kv8_slot(const Kv8Attn &a, int i, int lane) {
  constexpr int kAll = 1 << 30;
  const int G = a.Hq / a.Hkv;
  const Kv8Slot none{-1, 0, 0, 0, 0, {0, 0}, 0};
  if (a.B > 64) {
    const int b = kv8_find(a.B, lane, i,
                           [&](int x) { return kv8_tile_slot((int64_t)a.cu[x] * G, x, kRows); });
    if (b < 0) return none;
    const Kv8Rows rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
    const int64_t tiles = ((int64_t)rows.n * G + kRows - 1) / kRows;
    const int64_t tile = tiles - 1 - (i - kv8_tile_slot((int64_t)a.cu[b] * G, b, kRows));
    if (tile < 0 || tile >= tiles) return none;
    return {b, tile, 0, 1, kAll, rows, a.kv_len[b]};
  }
  int tiles = 0, before = 0, kv_len = 0;
  Kv8Rows rows{0, 0};
  if (lane < a.B) {
    rows = kv8_rows(a.cu[lane], a.cu[lane + 1], a.T);
    kv_len = a.kv_len[lane];
    tiles = (int)(((int64_t)rows.n * G + kRows - 1) / kRows);
    if (a.causal && a.window == 0)
      before = (int)kv8_min(kv8_max(kv8_len(kv_len, a.cache.max_pages) - rows.n, 0) * G / kRows, 1 << 24);
  }
  const auto more = [&](int x) {
    return __builtin_amdgcn_readlane(wave_upto(max(min(tiles + before - x, tiles), 0)), 63);
  };
  if (i >= more(0)) return none;
  int x = 0, past = tiles + before;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) past = max(past, __shfl_xor(past, off));
  past = __builtin_amdgcn_readfirstlane(past);
  while (past - x > 1) {
    const int half = x + (past - x) / 2;
    if (more(half) > i)
      x = half;
    else
      past = half;
  }
  const int rank = i - more(x + 1);
  const bool has = x >= before && x < before + tiles;
  const uint64_t like = __ballot(has);
  const bool mine = has && __popcll(like & ((uint64_t(1) << lane) - 1)) == rank;
  const int b = __builtin_ctzll(__ballot(mine));
  return {b, x - __builtin_amdgcn_readlane(before, b), 0, 1, kAll,
          {__builtin_amdgcn_readlane(rows.row0, b), __builtin_amdgcn_readlane(rows.n, b)},
          __builtin_amdgcn_readlane(kv_len, b)};
}

// A page's first DC channels (of DP) in LDS, and one wave's 32 rows.  (V's rows past them,
// up to a whole product's, are never written: nor are the channels that come of them.)
template <int DP, int DC>
struct Kv8Tile {
  static constexpr int kKStride = DC + 8, kVStride = kKv8Page + 8;  // halves; off the banks
  static constexpr int kSteps = DC / 16, kOut = (DC + 31) / 32;
  static constexpr int kKPage = kKv8Page * kKStride, kVPage = 32 * kOut * kVStride;
  static constexpr int kUnits = DC * kKv8Page / 16;  // 16 bytes each, of a page's K as of its V

  int b, h, len, first_page, pages;
  bool bad;  // more keys than the table has pages for

  bool in, empty;              // this lane's row is one; it sees no key
  int64_t out;                 // its number among all rows of all heads
  int key_lo, key_hi;          // the keys that it sees
  int all_lo, all_hi;          // that all of the wave's see
  int any_lo, any_hi;          // that some of them sees
  int key_at, value_at;        // its first halves of a page's K and V in LDS
  v8h q[kSteps];
  v16f o[kOut];
  float m, l;

  int part, parts;             // which of a tile's runs of pages this is

  // What the head's i-th workgroup takes; false where that is nothing.
  template <int kRows>
  __device__ __forceinline__ bool aim(const Kv8Attn &a, const Kv8Parts &p, int i, int head_k, int wave,
                                      int lane) {
    const int col = lane & 31, half = lane >> 5;
    const int G = a.Hq / a.Hkv;
    h = head_k;
    const Kv8Slot at = p.parts > 1 ? kv8_part<kRows>(a, p, i, lane) : kv8_slot<kRows>(a, i, lane);
    b = at.b;
    if (b < 0) return false;
    const int64_t tile = at.tile;
    const Kv8Rows rows = at.rows;
    const int64_t whole = at.kv_len;
    len = (int)kv8_len(whole, a.cache.max_pages);
    bad = whole > len;
    const int all = rows.n * G, row0 = (int)tile * kRows + 32 * wave;
    const int q0 = (int)tile * kRows / G, q1 = min((int)(tile + 1) * kRows - 1, all - 1) / G;
    const Kv8Span span = kv8_span(len, rows.n, q0, q1 - q0 + 1, a.causal, a.window);
    // even runs of pages
    const int count = span.p1 - span.p0;
    const int some_parts = max(min(at.parts, (int)(((int64_t)count + at.most - 1) / at.most)), 1);
    const int run = (count + some_parts - 1) / some_parts;
    part = at.part;
    parts = run == 0 ? 1 : (count + run - 1) / run;
    if (part >= parts) return false;
    first_page = span.p0 + part * run;
    pages = min(run, span.p1 - first_page);
    id = max(lookup(a, lane), 0);  // the first that something waits for

    const int row = row0 + col;
    in = row < all;
    const int some = in ? row : all - 1, qi = some / G, head = h * G + some % G;
    out = (int64_t)(rows.row0 + qi) * a.Hq + head;
    const uint16_t *qp = a.q + (int64_t)(rows.row0 + qi) * a.ldq + head * a.D;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const int d = 16 * st + 8 * half;
      v4u w = {0u, 0u, 0u, 0u};
      if (d < a.D) w = *reinterpret_cast<const v4u *>(qp + d);
      if (a.scale < 0.f) w ^= 0x80008000u;  // the factor of a score is not negative then
      q[st] = __builtin_bit_cast(v8h, w);
    }
    const int pos = len - rows.n + qi;
    empty = kv8_empty(a, len, pos, bad);
    key_hi = a.causal ? pos : len - 1;
    key_lo = a.window > 0 ? (int)kv8_max(pos - a.window + 1, 0) : 0;
    const int w0 = min(row0, all - 1) / G, w1 = min(row0 + 31, all - 1) / G;
    all_hi = a.causal ? len - rows.n + w0 : len - 1;
    any_hi = row0 >= all ? -1 : a.causal ? len - rows.n + w1 : len - 1;
    any_lo = a.window > 0 ? (int)kv8_max(0, len - rows.n + w0 - a.window + 1) : 0;
    all_lo = a.window > 0 ? (int)kv8_max(0, len - rows.n + w1 - a.window + 1) : 0;
    key_at = (16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3)) * kKStride +
             8 * half;
    value_at = col * kVStride + 8 * half;
    m = kNegInf;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    return true;
  }

  // Pages' numbers and scales are looked up 64 at a time, one to a lane: looked up when
  // they are needed, they would be two memory latencies in every page.
  int id;           // of the pages from 64 (j / 64) on: where codes are fetched
  float f, lg, iv;  // of the same pages, where scores become weights: factor of a score,
                    // value exponent and what undoes that
  __device__ __forceinline__ int lookup(const Kv8Attn &a, int j) const {
    if (j >= pages) return -1;
    return (int)kv8_page(a.cache.table, b, first_page + j, a.cache.max_pages, a.cache.num_pages);
  }
  // The first of page j's pages and heads in the pool (some page for one that it does not
  // have).
  __device__ __forceinline__ int64_t place(const Kv8Attn &a, int j, int lane) {
    if ((j & 63) == 0 && j > 0) id = max(lookup(a, j + lane), 0);
    return (int64_t)__builtin_amdgcn_readlane(id, j & 63) * a.Hkv + h;
  }
  __device__ __forceinline__ void scales(const Kv8Attn &a, int j, int lane, float fac) {
    if ((j & 63) != 0) return;
    const int page = lookup(a, j + lane);
    const int64_t ph = (int64_t)max(page, 0) * a.Hkv + h;
    f = factor(page < 0 || bad ? __builtin_nanf("") : a.cache.Ks[ph], fac);
    value_scale(page < 0 ? 0.f : a.cache.Vs[ph], lg, iv);
  }

  // A page's factor of a score: not 0, where what is masked would be NaN (all scores are 0
  // then, or as good as).
  static __device__ __forceinline__ float factor(float scale, float fac) {
    const float f = scale * fac;
    return f < 1e-30f ? 1e-30f : f;
  }

  // Scores of page j to weights.
  __device__ __forceinline__ void weights(int j, int lane, v16f (&x)[2], v8h (&w)[4]) {
    const int half = lane >> 5;
    float pf = lane_float(f, j & 63), plg = lane_float(lg, j & 63);
    const float piv = lane_float(iv, j & 63);
    const int token = (first_page + j) * kKv8Page;
    if (token < all_lo || token + kKv8Page - 1 > all_hi) {
      asm volatile("");  // a branch, not selects on every page
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = token + 32 * t + 16 * (i >> 3) + 8 * half + (i & 7);
          if (key < key_lo || key > key_hi) x[t][i] = kNegInf;
        }
      // a row that sees none of the page keeps out of its scales, which can be NaN
      if (key_hi < token || key_lo > token + kKv8Page - 1) {
        pf = 1.f;
        plg = 0.f;
      }
    }
    float sum;
    const auto all_weights = [&](auto exponent) {
      sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = exp2_fast(exponent(x[t][i]));
          sum += e;
          w[2 * t + (i >> 3)][i & 7] = (_Float16)e;
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));  // here, not among the products
    };
    const float off = plg - (m == kNegInf ? 0.f : m);  // no key yet
    all_weights([&](float s) { return __builtin_fmaf(s, pf, off); });
    // The largest exponent is looked for only where weights are too large, or have no
    // reference yet.
    if (__any(sum > kMostSum || m == kNegInf)) {
      asm volatile("");
      float most = kNegInf;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, x[t][i]);
      most = __builtin_fmaf(max_xor32(most), pf, plg);
      const float now = raise_ref(m, most);
      const float keep = m == now ? 1.f : exp2_fast(m - now);
      m = now;
      l *= keep;
#pragma unroll
      for (int t = 0; t < kOut; ++t) o[t] *= keep;
      const float ref = m == kNegInf ? 0.f : m, now_off = plg - ref;
      if (__any(fabsf(ref) > 0x1p24f)) {
        // Exponents so large are rounded by more than a weight's range: rounded as the largest
        // one was, none of them passes kMost.  (Here alone: for all scores it is 1 % slower.)
        asm volatile("");
        all_weights([&](float s) { return __builtin_fmaf(s, pf, plg) - ref; });
      } else {
        asm volatile("");
        all_weights([&](float s) { return __builtin_fmaf(s, pf, now_off); });
      }
    }
    l = __builtin_fmaf(sum, piv, l);
  }

  // Products in a row: O += V W where VALUES (w of a page, its V at vs), X = K Q where
  // SCORES (another page's K at ks).  Fragments come out of LDS kAhead products early.
  template <bool VALUES, bool SCORES>
  __device__ __forceinline__ void products(const _Float16 *vs, const v8h (&w)[4], const _Float16 *ks,
                                           v16f (&x)[2]) {
    constexpr int kV = VALUES ? 4 * kOut : 0, kS = SCORES ? 2 * kSteps : 0, kAhead = DP == 192 ? 3 : 6;
    const _Float16 *vp = vs + value_at, *kp = ks + key_at;
    auto fragment = [&](int i) {
      return i < kV ? *reinterpret_cast<const v8h *>(vp + 32 * (i % kOut) * kVStride + 16 * (i / kOut))
                    : *reinterpret_cast<const v8h *>(kp + 32 * ((i - kV) & 1) * kKStride + 16 * ((i - kV) >> 1));
    };
    if constexpr (SCORES) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
    }
    v8h ring[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ring[i] = fragment(i);
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int i = 0; i < kV + kS; ++i) {
      const v8h now = ring[i % kAhead];
      if (i < kV)
        o[i % kOut] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now, w[i / kOut], o[i % kOut], 0, 0, 0);
      else
        x[(i - kV) & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now, q[(i - kV) >> 1], x[(i - kV) & 1], 0, 0, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i + kAhead < kV + kS) {
        ring[i % kAhead] = fragment(i + kAhead);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
  }

  __device__ __forceinline__ void finish(const Kv8Attn &a, const Kv8Parts &p, int half) {
    l += __shfl_xor(l, 32);
    if (bad) l = __builtin_nanf("");  // also where the row sees none of the table's places
    if (!in) return;
    if (p.counts != nullptr && part == 0 && half == 0) p.counts[out] = empty ? -parts : parts;
    if (parts > 1) {
      const int64_t at = part * p.rows + out;
      if (half == 0) {
        p.m[at] = m;
        p.l[at] = l;
      }
#pragma unroll
      for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<v4f *>(p.o + at * DP + 32 * t + 2 * i + 4 * half) =
              v4f{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
      return;
    }
    const float scale = 1.f / l;
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
        *reinterpret_cast<v2u *>(a.Y + out * a.D + d) = y;
      }
    if (half == 0 && a.lse != nullptr) a.lse[out] = empty ? kNegInf : (m + log2f(l)) * kLn2;
  }

  // Where 16 codes (unit u of a page's K; V's are in order) come from, and where they go
  // in LDS, as fp16.
  static __device__ __forceinline__ int key_bytes(int u) {
    return DC == DP ? u * 16 : u / (DC / 16) * DP + u % (DC / 16) * 16;
  }
  static __device__ __forceinline__ int key_place(int u) {
    return u / (DC / 16) * kKStride + u % (DC / 16) * 16;
  }
  static __device__ __forceinline__ int value_place(int u) {
    return u / (kKv8Page / 16) * kVStride + u % (kKv8Page / 16) * 16;
  }
};

__device__ __forceinline__ void stage16(_Float16 *to, v4u w) {
  *reinterpret_cast<v8h *>(to) = kv8_halves(w[0], w[1]);
  *reinterpret_cast<v8h *>(to + 8) = kv8_halves(w[2], w[3]);
}

// One phase after another: every wave does scores, softmax and values of a page, and its
// part of the next page's codes, between two barriers.
template <int DP, int DC, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2) void kv8_tile_kernel(Kv8Attn a, Kv8Parts parts) {
  using Tile = Kv8Tile<DP, DC>;
  constexpr int kThreads = 64 * WAVES, kUnits = Tile::kUnits;
  constexpr int kLoads = (2 * kUnits + kThreads - 1) / kThreads;  // K's units, then V's
  static_assert(kUnits % 64 == 0, "whole waves");
  __shared__ __attribute__((aligned(16))) _Float16 ks[2][Tile::kKPage];
  __shared__ __attribute__((aligned(16))) _Float16 vs[2][Tile::kVPage];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Tile t;
  if (!t.template aim<32 * WAVES>(a, parts, blockIdx.x / a.Hkv, blockIdx.x % a.Hkv, wave, lane)) return;
  const float fac = fabsf(a.scale) * kLog2e;

  v4u code[kLoads];
  auto fetch = [&](int j) {
    const int64_t ph = t.place(a, j, lane);
    const __amdgpu_buffer_rsrc_t keys = make_rsrc(a.cache.Kc + ph * (DP * kKv8Page), DP * kKv8Page);
    const __amdgpu_buffer_rsrc_t values = make_rsrc(a.cache.Vc + ph * (DP * kKv8Page), DP * kKv8Page);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * kThreads + wave * 64;  // a wave's are all of one kind
      if (at < kUnits)
        code[u] = __builtin_amdgcn_raw_buffer_load_b128(keys, Tile::key_bytes(u * kThreads + tid), 0, 0);
      else if (at < 2 * kUnits)
        code[u] = __builtin_amdgcn_raw_buffer_load_b128(values, (u * kThreads + tid - kUnits) * 16, 0, 0);
    }
  };
  auto stage = [&](int to) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * kThreads + wave * 64;
      if (at < kUnits)
        stage16(ks[to] + Tile::key_place(u * kThreads + tid), code[u]);
      else if (at < 2 * kUnits)
        stage16(vs[to] + Tile::value_place(u * kThreads + tid - kUnits), code[u]);
    }
  };
  if (t.pages > 0) {
    fetch(0);
    stage(0);
  }
  for (int j = 0; j < t.pages; ++j) {
    __syncthreads();  // this page is there, and the one before is done with
    const bool more = j + 1 < t.pages;
    if (more) fetch(j + 1);
    t.scales(a, j, lane, fac);
    const int token = (t.first_page + j) * kKv8Page;
    if (token <= t.any_hi && token + kKv8Page > t.any_lo) {  // else no row of the wave sees it
      v16f x[2];
      v8h w[4];
      t.template products<false, true>(nullptr, w, ks[j & 1], x);
      t.weights(j, lane, x, w);
      t.template products<true, false>(vs[j & 1], w, nullptr, x);
    }
    if (more) stage((j + 1) & 1);
  }
  t.finish(a, parts, lane >> 5);
}

// LDS is as this wave has left it, and the other waves too.  (Global loads stay in flight.)
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Two teams of four waves, one of each to a SIMD, half a page apart: while one has the
// matrix cores (values of a page, scores of the next), the other has the vector units
// (softmax, codes to fp16), and at every barrier they change over.  With i counting the
// intervals between barriers, the first team has its products in even i and the second in
// odd i: scores of page j in 2 j and 2 j + 1, values in 2 j + 2 and 2 j + 3.  The first
// team brings K: page j + 1 in interval 2 j + 1, over page j - 1, last read in 2 j - 1.
// The second brings V: page j + 1 in interval 2 j + 2, over page j - 1, last read in
// 2 j + 1.  Each therefore has two stages.  (On 8192 tokens of 72 heads 256 rows took 1430 us
// one phase after another where the teams took 1235; an interval is some 2000 cycles, evenly
// matched.)
template <int DP, int DC>
__global__ __launch_bounds__(512, 2) void kv8_pair_kernel(Kv8Attn a, Kv8Parts parts) {
  using Tile = Kv8Tile<DP, DC>;
  constexpr int kUnits = Tile::kUnits, kLoads = (kUnits + 255) / 256;
  __shared__ __attribute__((aligned(16))) _Float16 ks[2][Tile::kKPage];
  __shared__ __attribute__((aligned(16))) _Float16 vs[2][Tile::kVPage];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, mine = tid & 255;
  const bool second = wave >= 4;
  Tile t;
  if (!t.template aim<256>(a, parts, blockIdx.x / a.Hkv, blockIdx.x % a.Hkv, wave, lane)) return;
  const float fac = fabsf(a.scale) * kLog2e;

  v4u code[kLoads];
  const uint8_t *pool = second ? a.cache.Vc : a.cache.Kc;
  auto fetch = [&](int j) {
    const int64_t ph = t.place(a, j, lane);
    const __amdgpu_buffer_rsrc_t page = make_rsrc(pool + ph * (DP * kKv8Page), DP * kKv8Page);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (u * 256 + (wave & 3) * 64 < kUnits)
        code[u] = __builtin_amdgcn_raw_buffer_load_b128(
            page, second ? (u * 256 + mine) * 16 : Tile::key_bytes(u * 256 + mine), 0, 0);
  };
  auto stage = [&](int j) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (u * 256 + (wave & 3) * 64 < kUnits)
        stage16(second ? vs[j & 1] + Tile::value_place(u * 256 + mine)
                       : ks[j & 1] + Tile::key_place(u * 256 + mine), code[u]);
  };
  const int n = t.pages;
  if (n > 0) {
    v16f x[2];
    v8h w[4];
    fetch(0);
    stage(0);
    if (n > 1) fetch(1);
    meet();
    if (second) meet();
    auto soft = [&](int j, bool more) {
      t.scales(a, j, lane, fac);
      t.weights(j, lane, x, w);
      if (more) {
        stage(j + 1);
        if (j + 2 < n) fetch(j + 2);
      }
    };
    t.template products<false, true>(nullptr, w, ks[0], x);
    meet();
    for (int j = 0; j + 1 < n; ++j) {
      soft(j, true);
      meet();
      t.template products<true, true>(vs[j & 1], w, ks[(j + 1) & 1], x);
      meet();
    }
    soft(n - 1, false);
    meet();
    t.template products<true, false>(vs[(n - 1) & 1], w, nullptr, x);
    if (!second) meet();
  }
  t.finish(a, parts, half);
}

}  // namespace detail

// Workgroups of a key head: with shared tiles twice as many as run at a time (the first
// tiles' pages may be none, so the last ones' sum may be twice the even one) and one for
// every tile.
static int kv8_workgroups(const Kv8Attn &a, const Kv8Parts &p, int rows) {
  const int tiles = (int)kv8_tile_slots((int64_t)a.T * (a.Hq / a.Hkv), a.B, rows);
  return p.parts > 1 ? tiles + 2 * p.groups / a.Hkv + 1 : tiles;
}
template <int DP, int DC = DP, int WAVES = 4>
static hipError_t tile_launch(const Kv8Attn &a, Kv8Parts p, hipStream_t st) {
  p.slots = kv8_workgroups(a, p, 32 * WAVES);
  detail::kv8_tile_kernel<DP, DC, WAVES><<<(unsigned)p.slots * a.Hkv, 64 * WAVES, 0, st>>>(a, p);
  return hipGetLastError();
}
template <int DP, int DC = DP>
static hipError_t pair_launch(const Kv8Attn &a, Kv8Parts p, hipStream_t st) {
  p.slots = kv8_workgroups(a, p, 256);
  detail::kv8_pair_kernel<DP, DC><<<(unsigned)p.slots * a.Hkv, 512, 0, st>>>(a, p);
  return hipGetLastError();
}

hipError_t launch_kv8_tiles(const Kv8Attn &a, int rows, const Kv8Parts &p, hipStream_t st) {
  // The widths that a head's 16 channels make, but for the narrowest and the widest: 4 x
  // 2048 tokens take the same 238 us with 16 heads of 208 as of 256 channels, and with 32
  // heads of 16, 32, 48 and 64 channels 95, 98, 101 and 102, mostly for the softmax.
  switch ((a.D + 15) / 16) {
    case 5: return tile_launch<96, 80>(a, p, st);
    case 6: return tile_launch<96>(a, p, st);
    case 7: return rows == 256 ? pair_launch<128, 112>(a, p, st) : tile_launch<128, 112>(a, p, st);
    case 8: return rows == 256 ? pair_launch<128>(a, p, st) : tile_launch<128>(a, p, st);
    case 9: return pair_launch<192, 144>(a, p, st);
    case 10: return pair_launch<192, 160>(a, p, st);
    case 11: return pair_launch<192, 176>(a, p, st);
    case 12: return pair_launch<192>(a, p, st);
    default: return a.D <= 64 ? tile_launch<64>(a, p, st) : tile_launch<256>(a, p, st);
  }
}

}  // namespace ot
