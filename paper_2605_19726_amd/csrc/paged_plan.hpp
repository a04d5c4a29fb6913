// Arithmetic of the paged key-value cache that host and kernels share: division by a page size, and which workgroup of the
// single-token attention takes which tiles.  No HIP in here: the CPU tests compile it as it is.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define BASA_HD __host__ __device__ inline
#else
#define BASA_HD inline
#endif

namespace basa {

// n / d for 0 <= n < 2^31 by one multiplication: with l = ceil(log2 d) and mul = floor(2^32 (2^l - d) / d) + 1 the quotient is
// (floor(mul n / 2^32) + n) >> l (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994).  The
// sum stays below 2^32, since mul <= 2^32 and n < 2^31.
struct FastDiv {
  uint32_t d, mul, shift;
  BASA_HD uint32_t div(uint32_t n) const { return ((uint32_t)(((uint64_t)mul * n) >> 32) + n) >> shift; }
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f;
  f.d = d;
  f.shift = 0;
  while ((1ull << f.shift) < d) ++f.shift;
  f.mul = (uint32_t)((((1ull << f.shift) - d) << 32) / d + 1);
  return f;
}

// ---- single-token attention: work in a row, cut into equal runs -------------------------------------
// A workgroup takes the tokens of one (sequence, KV head, run of query heads) in steps of kDecodeStep, a tile of them per wave.
// All of a call, in the order sequence, head, token, lie on one axis: a (sequence, head) has place for its steps, at least one (also an
// empty one: someone has to write its rows), behind kDecodeLead places for what it costs to begin with it.  The axis of `total` places is
// cut into runs of equal length; workgroup w takes what lies in [w run, (w + 1) run).
constexpr int kDecodeTile = 32, kDecodeWaves = 4, kDecodeStep = kDecodeTile * kDecodeWaves;
constexpr int kDecodeLead = 1;
BASA_HD int decode_steps(int len) { return len <= kDecodeStep ? 1 : (len + kDecodeStep - 1) / kDecodeStep; }
BASA_HD int decode_places(int len) { return decode_steps(len) + kDecodeLead; }
// The length of a run: two workgroups fit a compute unit (bf16 d = 64: four, f32 d = 64: three), so short rows are cut into as many runs as there is
// room for at once.  Where those would be longer than 24 steps there are more, down to 8 steps, so that a workgroup that is done early is
// followed by another; 2048 at most.  That pays for long rows of pages stored token by token, and costs elsewhere.  Main kernel + join, one
// round -> runs of 8 and more, (sequence, head) of d = 128 in bf16 unless said; token by token: 512 of 8000 to 60000 tokens 968 + 4.2 -> 943 + 5.5
// us, 128 of 65536 713 + 4.1 -> 681 + 4.5, 512 of 3000 at d = 64 76 + 4.0 -> 70 + 4.2, 2048 of 3900 to 4000 617 + 5.0 -> 655 + 6.0, 1024 of 2000 163 + 4.0 ->
// 179 + 4.6; head by head: 512 of 8000 to 60000 906 + 4.2 -> 926 + 5.5, 128 of 65536 660 + 4.1 -> 671 + 4.5, 1024 of 2000 161 + 4.0 -> 172 + 4.4, f32 512 of 3000
// 238 + 4.1 -> 270 + 4.2; one sequence of 128K, 8 heads (17 steps, one round either way): 86.6 + 4.8, in runs of 8 88.7 + 5.8.
constexpr int kDecodeOneRound = 512, kDecodeMost = 2048, kDecodeLongRun = 24, kDecodeShortRun = 8;
BASA_HD int decode_run(int total) {          // total < 2^31 - kDecodeMost
  const int one = (total + kDecodeOneRound - 1) / kDecodeOneRound, many = (total + kDecodeMost - 1) / kDecodeMost;
  return one <= kDecodeLongRun ? one : many > kDecodeShortRun ? many : kDecodeShortRun;
}
// What lies in a run of a (sequence, head) whose first place is `first`: steps [t0, t1), none if t1 <= t0.
struct DecodePiece { int t0, t1; };
BASA_HD DecodePiece decode_piece(int first, int steps, int group, int run, int lead = kDecodeLead) {
  const int64_t begin = (int64_t)group * run - first - lead, end = begin + run;
  DecodePiece p;
  p.t0 = begin > 0 ? (int)(begin < steps ? begin : steps) : 0;
  p.t1 = end < steps ? (end > 0 ? (int)end : 0) : steps;
  return p;
}
// A run holds at most two pieces that are not whole: the end or middle of one that began before it, which has place 0 of the run's two
// partial results, and the beginning of one that goes on behind it, place 1.
BASA_HD int decode_part(DecodePiece p, int group) { return 2 * group + (p.t0 == 0 ? 1 : 0); }
// The groups that have steps of it: first and last.
BASA_HD int decode_first_group(int first, int run, int lead = kDecodeLead) { return (first + lead) / run; }
BASA_HD int decode_last_group(int first, int steps, int run, int lead = kDecodeLead) { return (first + lead + steps - 1) / run; }
// Workgroups of a call of up to `most` places, whatever the lengths turn out to be.
inline int decode_groups(int64_t most) { return (int)(most < kDecodeMost ? most : kDecodeMost); }

// ---- several new tokens of every sequence -----------------------------------------------------------
// The same axis for attention whose rows are (new token, query head) pairs: a (sequence, KV head) has a unit for every `tile` of its rows, none if
// there are none; the units lie in the order head, sequence, tile, each with places as above, for steps of `step` tokens.
BASA_HD constexpr int tree_lead(int step) { return step < kDecodeStep ? kDecodeStep / step : 1; }
BASA_HD int tree_steps(int len, int step) { return len <= step ? 1 : (len + step - 1) / step; }
BASA_HD int tree_units(int rows, int tile) { return (rows + tile - 1) / tile; }
// Rows [from, to) of a packed batch of `tokens` rows, of what it has of them: the first, and how many.  Less than none: offsets that do not ascend.
struct PackedRows { int row0, n; };
BASA_HD PackedRows packed_rows(int from, int to, int tokens) {
  const int first = from > 0 ? from : 0, last = to > 0 ? to : 0, row0 = first < tokens ? first : tokens;
  return {row0, (last < tokens ? last : tokens) - row0};
}
// What 32 drafted tokens from `at` on (negative: tokens of the context, which all see) the token `t` of a chain sees: those up to itself.
BASA_HD uint32_t chain_bits(int t, int at) {
  const int count = t - at + 1;
  return count <= 0 ? 0u : count >= 32 ? ~0u : (1u << count) - 1u;
}
// The same of the masks of a tree: the 64-bit words that hold bits at / 64 and at / 64 + 1 (zero where there is none; of at < 0: `low` is word 0).
BASA_HD uint32_t tree_bits(uint64_t low, uint64_t high, int at) {
  if (at <= -32) return ~0u;
  if (at < 0) return (uint32_t)(low << -at) | ((1u << -at) - 1u);
  const int s = at & 63;
  return (uint32_t)(s > 32 ? (low >> s) | (high << (64 - s)) : low >> s);
}

}  // namespace basa
