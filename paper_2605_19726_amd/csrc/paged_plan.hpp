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
BASA_HD int64_t decode_steps(int64_t len) { return len <= kDecodeStep ? 1 : (len + kDecodeStep - 1) / kDecodeStep; }
BASA_HD int64_t decode_places(int64_t len) { return decode_steps(len) + kDecodeLead; }
constexpr int kDecodeFew = 512, kDecodeMost = 3072, kDecodeLongRun = 32;
BASA_HD int64_t decode_run(int64_t total) {
  const int64_t few = (total + kDecodeFew - 1) / kDecodeFew, many = (total + kDecodeMost - 1) / kDecodeMost;
  return few <= kDecodeLongRun ? few : many > kDecodeLongRun ? many : kDecodeLongRun;
}
// What lies in a run of a (sequence, head) whose first place is `first`: steps [t0, t1), none if t1 <= t0.
struct DecodePiece { int64_t t0, t1; };
BASA_HD DecodePiece decode_piece(int64_t first, int64_t steps, int64_t group, int64_t run) {
  const int64_t begin = group * run - first - kDecodeLead, end = begin + run;
  DecodePiece p;
  p.t0 = begin > 0 ? begin : 0;
  p.t1 = end < steps ? end : steps;
  return p;
}
// A run holds at most two pieces that are not whole: the end or middle of one that began before it, which has place 0 of the run's two
// partial results, and the beginning of one that goes on behind it, place 1.
BASA_HD int64_t decode_part(DecodePiece p, int64_t group) { return 2 * group + (p.t0 == 0 ? 1 : 0); }
// The groups that have steps of it: first and last.
BASA_HD int64_t decode_first_group(int64_t first, int64_t run) { return (first + kDecodeLead) / run; }
BASA_HD int64_t decode_last_group(int64_t first, int64_t steps, int64_t run) { return (first + kDecodeLead + steps - 1) / run; }
// Workgroups of a call of up to `total` places, whatever the lengths turn out to be.
inline int decode_groups(int64_t most) {
  const int64_t n = most < kDecodeMost ? most : kDecodeMost;
  return (int)n;
}

}  // namespace basa
