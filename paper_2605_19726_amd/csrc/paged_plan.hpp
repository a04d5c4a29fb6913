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
BASA_HD DecodePiece decode_piece(int first, int steps, int group, int run) {
  const int64_t begin = (int64_t)group * run - first - kDecodeLead, end = begin + run;
  DecodePiece p;
  p.t0 = begin > 0 ? (int)(begin < steps ? begin : steps) : 0;
  p.t1 = end < steps ? (end > 0 ? (int)end : 0) : steps;
  return p;
}
// A run holds at most two pieces that are not whole: the end or middle of one that began before it, which has place 0 of the run's two
// partial results, and the beginning of one that goes on behind it, place 1.
BASA_HD int decode_part(DecodePiece p, int group) { return 2 * group + (p.t0 == 0 ? 1 : 0); }
// The groups that have steps of it: first and last.
BASA_HD int decode_first_group(int first, int run) { return (first + kDecodeLead) / run; }
BASA_HD int decode_last_group(int first, int steps, int run) { return (first + kDecodeLead + steps - 1) / run; }
// Workgroups of a call of up to `most` places, whatever the lengths turn out to be.
inline int decode_groups(int64_t most) { return (int)(most < kDecodeMost ? most : kDecodeMost); }

}  // namespace basa
