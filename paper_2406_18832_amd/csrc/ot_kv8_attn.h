// What the two attention kernels over the 8-bit cache share.
//
// The softmax in one pass.  With x_j = log2(e) scale q.K_j, a row keeps a
// reference m, L = sum_j 2^(x_j + l_j - m) 2^(-l_j) and O = sum_j 2^(x_j + l_j - m) c_j,
// where a value V_j = 2^(l_j) c_j is a code c_j times its page's scale 2^(l_j): the
// value scale costs nothing there, as x_j + l_j is one fused multiply-add from the
// product of codes and queries.  O / L is the row's result; m and L are fp32.
//
// The weights 2^(x_j + l_j - m) are an operand of the matrix cores in fp16 (half a
// step is 2^-11 of a weight).  m is set kSet binades under the largest exponent and stays
// until a weight would pass 2^kMost: O and L are scaled anew a few times in a row's life,
// and fp16's normal numbers reach 2^-22 of the largest weight.  Below them a weight is off
// by at most 2^-33 of the largest; with a code of up to 127 that is 2^-26 of a step of the
// page with the largest, whose own values are only known to half a step.  (But for a page
// of zeros, whose values are exact: there l_j is the least that a scale has.)  L sums the
// fp32 weights.  Of the matrix cores' fast types fp16 rounds the least; with fp32 operands
// the second product would run at the rate of the fp32 instructions, a sixteenth.  The
// rounding adds to Y's own: 64 single tokens of 40 heads are off by 2.6 10^-4 of Y's norm, with
// weights in fp32 by 2.1.  (Tiles, whose time goes by vector instructions, look for the largest
// exponent only where the sum of a lane's weights of a page, none of which is larger than
// it, passes kMostSum or a row has no m yet.)
//
// Which weight belongs to which token.  S^T = K Q^T has tokens as the MFMA's rows
// and queries as its columns, and leaves a lane with weights of one query alone,
// which are, in this order, the operand of O^T = V^T P^T as long as K's row r stands
// for the right token: no weight changes its lane.
#pragma once

#include "ot_kv8.h"

namespace ot {
namespace detail {

constexpr float kSet = 8.f, kMost = 15.f, kMostSum = 32768.f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A value scale's exponent and what undoes it: a page of zeros (scale 0) counts as scale
// 2^-31, below which no page's is (fp16's least number over 127).  With scale 1 a zero page
// with a key 14 binades ahead of the others', whose values are of 1e-3 and their scales of
// 2^-17, would take the others' weights out of fp16's normal numbers.  A NaN goes by the exponent alone, which reaches the rows that see the page
// and no others.
__device__ __forceinline__ void value_scale(float s, float &lg, float &inv) {
  const float v = s == 0.f ? 0x1p-31f : s;
  lg = __builtin_amdgcn_logf(v);  // log2
  inv = v == v ? 1.f / v : 1.f;
}

__device__ __forceinline__ v2h pack_half(float a, float b) {
  return v2h{(_Float16)a, (_Float16)b};  // each to nearest even
}

// A row's reference where `most` is the largest exponent of some keys and m the reference
// so far: most - kSet where that is larger, or most itself where fp32's numbers are so far
// apart (from exponents of 2^24 on) that the difference would pass kMost.
__device__ __forceinline__ float raise_ref(float m, float most) {
  const float now = fmaxf(m, most - kSet);
  return most - now > kMost ? most : now;
}

// The maximum over the lanes of one query: xor 16 and xor 32, or xor 32 alone.  A swap
// of a register's rows with those of its copy leaves each lane the other's value.
__device__ __forceinline__ float max_xor16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float max_xor32(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float lane_float(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// How the pages of a batch are shared out between workgroups.  An item is a run of
// at most `chunk` pages of one sequence; every workgroup works out from the lengths
// how many there are (their sizes are even whatever the lengths: a long sequence
// among short ones has many) and which one is its own.
struct Kv8Item {
  int b, index, chunk;  // sequence (-1: none), which of its items, pages per item
  int first, count;     // its sequence's first item and their number
};

// Sequence b's pages and rows, by one lane.
struct Kv8Seq {
  Kv8Rows rows;
  int64_t len;
  Kv8Span span;
  bool bad;  // more keys than its table has pages for
};
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8Attn &a, int b) {
  Kv8Seq s;
  s.rows = kv8_rows(a.cu[b], a.cu[b + 1], a.T);
  const int64_t len = a.kv_len[b];
  s.len = kv8_len(len, a.cache.max_pages);
  s.bad = len > s.len;
  s.span = kv8_span(s.len, s.rows.n, 0, s.rows.n, a.causal, a.window);
  return s;
}
// Whether a row at position pos of len keys sees none, and is 0.  Where the sequence has more
// keys than its table has pages for (bad), len and with it pos are not its own: its rows are
// NaN, also those before position 0.
__device__ __forceinline__ bool kv8_empty(const Kv8Attn &a, int64_t len, int64_t pos, bool bad) {
  return !bad && (len == 0 || (a.causal && pos < 0));
}
// Pages that count in the sharing: at least one, which writes the rows that see no key.
__device__ __forceinline__ int kv8_shared_pages(const Kv8Seq &s) {
  return s.rows.n == 0 ? 0 : max(s.span.p1 - s.span.p0, 1);
}

// Inclusive sums along the lanes (DPP: no LDS); lane 63 has the wave's.
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ int wave_upto(int v) {
  v = dpp_add<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);  // row_bcast:15 to rows 1 and 3
  return dpp_add<0x143, 0xc>(v);  // row_bcast:31 to rows 2 and 3
}

// Item x.  Pages per item: the fewest, but `least`, that make at most `wanted` items (as
// many as run at a time) where that many leave each sequence one; else those of which
// `wanted` make all pages.  Items are then at most `wanted` and one per sequence.  wanted
// 0: every sequence is one item.
__device__ __forceinline__ Kv8Item kv8_item(const Kv8Attn &a, int lane, int x, int wanted,
                                            int least) {
  if (wanted == 0) return {x < a.B ? x : -1, 0, 1 << 30, x, 1};
  int pages = lane < a.B ? kv8_shared_pages(kv8_seq(a, lane)) : 0;
  int64_t total = __builtin_amdgcn_readlane(wave_upto(pages), 63);
  for (int b = 64; b < a.B; b += 64)
    total += __builtin_amdgcn_readlane(
        wave_upto(b + lane < a.B ? kv8_shared_pages(kv8_seq(a, b + lane)) : 0), 63);
  int chunk = (int)kv8_max(least, (total + wanted - 1) / wanted);
  if (a.B <= 64 && a.B <= wanted) {
    // between these two: with the larger, rounding up cannot make too many
    int most = (int)kv8_max(chunk, wanted > a.B ? (total + wanted - a.B - 1) / (wanted - a.B) : 1 << 30);
    const auto items = [&](int c) {
      return __builtin_amdgcn_readlane(wave_upto((int)((unsigned)(pages + c - 1) / (unsigned)c)), 63);
    };
    while (chunk < most) {
      const int half = chunk + (most - chunk) / 2;
      if (items(half) <= wanted)
        most = half;
      else
        chunk = half + 1;
    }
  }
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (b0 > 0) pages = b0 + lane < a.B ? kv8_shared_pages(kv8_seq(a, b0 + lane)) : 0;
    const int own = (int)((unsigned)(pages + chunk - 1) / (unsigned)chunk);
    const int upto = wave_upto(own);
    const uint64_t past = __ballot(before + upto > x);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      const int count = __builtin_amdgcn_readlane(own, at);
      const int first = before + __builtin_amdgcn_readlane(upto, at) - count;
      return {b0 + at, x - first, chunk, first, count};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, chunk, 0, 0};
}

// A row's partial result in the workspace: m, L and O[D] (fp32).
__device__ __forceinline__ int64_t kv8_partial(int64_t item, int64_t h, int64_t row, int64_t Hkv,
                                               int64_t rows) {
  return (item * Hkv + h) * rows + row;
}

}  // namespace detail

// Up to so many query rows to a key head and sequence the kernel for few rows runs.
constexpr int64_t kFewRows = 32;

// The kernel for few rows: 16-row tiles that a workgroup takes (two, where a wave's
// registers hold them: 117 sequences of 169-5610 keys of 2 x 24 heads of 144 channels 88 us
// against 118), and the workgroups that a CU holds.
constexpr int kv8_decode_tiles(int dp, int64_t rows) { return rows > 16 && dp <= 192 ? 2 : 1; }
constexpr int kv8_decode_waves(int dp, int tiles) {
  if (dp > 128) return dp == 192 && tiles == 1 ? 2 : 1;
  return tiles == 2 ? 2 : dp <= 64 ? 4 : 3;
}

// Partial results of a split launch: `items` runs of pages, `rows` rows to each key
// head.  spans [B] says which items a sequence has.
struct Kv8Split {
  int wanted, least;  // as kv8_item; wanted 0: no split
  int64_t items, rows;
  float *m, *l, *o;
  int2 *spans;
};

hipError_t launch_kv8_decode(const Kv8Attn &a, const Kv8Split &s, hipStream_t st);
hipError_t launch_kv8_combine(const Kv8Attn &a, const Kv8Split &s, hipStream_t st);

// A launch of tiles in which one's pages are shared between up to `parts` workgroups,
// `least` pages and more to each; `groups` of them run at a time, each key head has
// `slots`.  rows: all query rows, T Hq; for each of them how many parts it has, and part
// by part m, L and O [Dp].
struct Kv8Parts {
  int parts, least, groups, slots;
  int whole;  // pages up to which a tile is not split
  int64_t rows;
  int *counts;  // nullptr: one part
  float *m, *l, *o;
};
hipError_t launch_kv8_tiles(const Kv8Attn &a, int rows, const Kv8Parts &p, hipStream_t st);
hipError_t launch_kv8_join(const Kv8Attn &a, const Kv8Parts &p, hipStream_t st);

}  // namespace ot
