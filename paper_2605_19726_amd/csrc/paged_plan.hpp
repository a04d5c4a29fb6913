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

// ---- single-token attention: tiles in a row, cut into equal runs -----------------------------------
// A tile is kDecodeTile cached tokens of one (sequence, KV head, run of query heads).  All tiles of a call, in the order sequence,
// head, token, make one row of `total` tiles that is cut into runs of run_tiles(total, groups); workgroup w takes the tiles
// [w run, (w + 1) run).  A sequence has at least one tile, also an empty one: someone has to write its rows.
constexpr int kDecodeTile = 32;
constexpr int kDecodeWaves = 4;              // waves of a workgroup: every one takes each fourth tile
BASA_HD int64_t decode_tiles(int64_t len) { return len <= kDecodeTile ? 1 : (len + kDecodeTile - 1) / kDecodeTile; }
// A multiple of the waves: a run that is not leaves some of them idle in its last step.
BASA_HD int64_t decode_run(int64_t total, int groups) {
  return (total + (int64_t)groups * kDecodeWaves - 1) / ((int64_t)groups * kDecodeWaves) * kDecodeWaves;
}
// A run can hold the end of one piece that began before it, and the beginning of one that goes on behind it, pieces that lie
// in it whole between them: two partial results at most.  A piece that covers the run's first tile has place 0.
BASA_HD int decode_part(int64_t first_tile, int64_t group, int64_t run) {
  return (int)(2 * group + (first_tile > group * run ? 1 : 0));
}

}  // namespace basa
