// Attention of several new tokens of every sequence, a tree or a chain of drafted ones, over its pages of the key-value cache (gfx950).
//
// A sequence holds `len` tokens, of which the last n are the new ones (their rows of q; keys and values are in the pages); base = len - n.  Token t sees
// every token before base, and new token j if bit j of its mask is set (a chain: j <= t).  Rows of a KV head: (t, h), n x group of them.  For
// a row:  s_j = q . k_j,  m = max s_j,  o = sum_j e^((s_j - m) / sqrt(d)) v_j / sum_j e^((s_j - m) / sqrt(d)),  lse = m / sqrt(d) + ln sum, over the tokens
// that it sees.  One pass over the tokens with a running maximum and sum per row.
//
// Bound by the memory up to some 64 rows of a KV head (bf16), by the matrix and vector units and the card's power from 200 on.  What carries it:
//   - All rows of a KV head share a token's K and V: a workgroup has a tile of 32 to 256 of them, a wave 32 (f32: 16), and the tokens come by in steps of 32 (16) through a
//     ring in the LDS, which requests to memory fill without registers (32 sequences of 1000 to 16000 tokens, 8 to 24 new ones, 32 heads on 8, d = 128: 698 MB in 144 us,
//     4.85 TB/s; 16 rows to a wave, its operands from memory: 180).
//   - S^T = K Q^T and O^T = V^T P^T: a lane has the same row in the scores, the weights and the output, so that weights are operands where they are, and the maximum and
//     the sum of a row are two lanes' (four).
//   - Weights enter the second product as two bf16 numbers, the upper half of the f32 and the rest: three products of matrix units for two of the formula, and the only rounding to
//     8 bits is the output's.  (131072 tokens, 64 new ones, 256 rows: 229 us, 900 TF executed of the 1276 that a large product of matrices runs at.  48% of the cycles
//     the matrix units work, and in 42% there are other vector instructions: they follow each other.  The next step's scores during this one's products, waves of
//     different priority, one barrier to two or four steps leave the time as it is (225 to 240).  There are 1.13 LDS instructions to a product; a wave of 64 rows, which
//     would halve them, has not been tried.)
//   - Work is cut on one axis (paged_plan.hpp): KV head by KV head, in each the sequences, in each the tiles of rows, each with a place for every step and some for what a
//     piece costs by itself; every workgroup finds its run of places from the lengths.  Pieces are added up by a second kernel where their L2 has them.
#include <algorithm>
#include <climits>
#include <type_traits>
#include "common.hpp"
#include "paged_plan.hpp"

namespace basa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(3))) char* lds_cptr_t;
typedef __attribute__((address_space(3))) uintx4* lds_chunk_ptr_t;
typedef __attribute__((address_space(3))) short4v* lds_quad_ptr_t;

struct TreeArgs {
  const char *q, *k, *v;
  int64_t q_t, q_h;                         // strides in bytes
  int64_t k_h, v_h;
  uint32_t k_b, k_l, v_b, v_l;              // of a page and of a token, in units of 2^unit bytes
  int unit;
  const int32_t *table, *lens, *cu;
  int64_t table_stride;
  int n, tokens, heads_kv, group, pages;    // sequences; rows of q
  int row_tokens;                           // tokens a table row has room for
  FastDiv page, per_token;                  // per_token: division by the group
  const int64_t* slots;                     // or null: every new token is in its pages
  int64_t all_slots;
  const uint64_t* masks;                    // or null: chains
  int64_t mask_stride;
  int words;
  char* out;
  int64_t out_t, out_h;                     // in bytes
  float* lse;                               // [tokens][heads_q] or null
  int groups;                               // workgroups, a multiple of 8
  int runs;                                 // at most so many runs (cut by runs)
  int* first_place;                         // workspace, of more than kPlanBatch sequences: [n + 1] first place of each for one head, then how many there are
  int* cut_of;                              // workspace: [tokens][heads_q] first and last run that have steps of a row, and its place in the tile; -1: one run has all
  float* part_o;                            // [2 runs][tile][d], not normalised
  float2* part_ml;                          // [2 runs][tile] maximum in units of the exponent, sum
  float scale_log2e;                        // log2 e / sqrt(d)
};
constexpr int kPlanBatch = 512;             // up to this many sequences every wave sums up the lengths by itself
constexpr int kWindow = 256;                // tokens whose places in the cache are in the LDS, twice
// How far a row's scores, in units of the exponent, may rise above the maximum that its weights refer to before these are scaled: weights up to 2^8 are as exact as
// weights up to 1.  Sums of large values could be no number for it where they are one with weights up to 1: from kLarge on they are made again with those.  (Below it
// those of all parts of a row, 1024 at most, are a number.)
constexpr float kRise = 8.f, kLarge = 0x1p117f;

// n < 0: the offsets do not ascend.  Then nothing is done, since rows that several sequences have could be more than the axis has places for.
struct Sequence { int len, row0, n; };
__device__ __forceinline__ Sequence sequence_of(const TreeArgs& a, int b) {
  const PackedRows rows = packed_rows(a.cu[b], a.cu[b + 1], a.tokens);
  return {min(max(a.lens[b], 0), a.row_tokens), rows.row0, rows.n};
}
constexpr int kMostRuns = 1024, kMostRows = 256;
__device__ __forceinline__ int pack_cut(int first, int last, int row) { return first + kMostRuns * (last + kMostRuns * row); }
__device__ __forceinline__ int sum_of(int x, int y) { return x + y; }
template <int kOff>
__device__ __forceinline__ float pair_max(float v) {
  uint32_t x, y;
  lane_pair<kOff>(__float_as_uint(v), x, y);
  return fmaxf(__uint_as_float(x), __uint_as_float(y));
}
template <int kOff>
__device__ __forceinline__ float pair_sum(float v) {
  uint32_t x, y;
  lane_pair<kOff>(__float_as_uint(v), x, y);
  return __uint_as_float(x) + __uint_as_float(y);
}
__device__ __forceinline__ float exponent_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float factor_of(float m, float top) { return __builtin_amdgcn_exp2f(m - exponent_base(top)); }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : fmaf(m, 0.6931471805599453f, __logf(l)); }
__device__ __forceinline__ floatx4 normalised(floatx4 o, float sum) { return sum == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / sum); }
template <bool kBf16>
__device__ __forceinline__ void store4(char* at, floatx4 o) {
  if constexpr (kBf16) {
    bf16x4 t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (__bf16)o[e];
    *reinterpret_cast<bf16x4*>(at) = t;
  } else {
    *reinterpret_cast<floatx4*>(at) = o;
  }
}
// 16 bytes from memory for every lane, side by side into the LDS.  Written in assembly, without a register for its result: the compiler would wait for all of
// these before it reads the LDS or meets a barrier; the waits stand where the ring needs them.  As a stream that no cache keeps: 8 new tokens of 32 sequences 130 us, and 148
// without that; level where a KV head has several tiles and reads its rows as often.  m0, the place in the LDS, is an operand, so that the compiler knows when it changes; between
// its write and such a load there has to be an instruction.
__device__ __forceinline__ void to_lds(const char* from, uint32_t at) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "{m0}"(at) : "memory");
}
__device__ __forceinline__ void word_to_lds(const void* from, uint32_t at) {      // 4 bytes for every lane
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "{m0}"(at) : "memory");
}
// Everyone's LDS operations are done before anyone goes on.  Requests by to_lds that are under way stay so.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(lds_cptr_t)p; }
__device__ __forceinline__ uintx4 lds_chunk(uint32_t at) { return *(lds_chunk_ptr_t)(uintptr_t)at; }
__device__ __forceinline__ bf16x4 lds_turned(uint32_t at) {
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad_ptr_t)(uintptr_t)at));
}

// Whether there are tokens of a step that the lane's row does not see, and bits of those that it does.
struct Seen { bool masked; uint32_t bits; };

// What a wave does with a step's tokens in the LDS for its rows.  Row of a lane: its column of the matrix instruction.
template <bool kBf16, int kD> struct Rows;

// bf16: 32 rows, 32x32x16 instructions.  S^T = K Q^T: lane (h, r) of the A operand holds chunk 2 c + h of token r at step c.  Of the result lane (h, n) holds
// tokens 8 q + 4 h + j (register 4 q + j) of row n: the B operand of O^T += V^T P^T for tokens 16 u .. 16 u + 15, if token 16 u + 8 w + 4 h + j stands at place
// 8 h + 4 w + j of the sum.  The A operand in that order: the transposing read gives lane i of 16 column i of the four rows that they address.
template <int kD>
struct Rows<true, kD> {
  static constexpr int kRows = 32, kTokens = 32, kKSteps = kD / 16, kBlocks = kD / 32, kRowBytes = kD * 2, kChunks = kRowBytes / 16;
  uintx4 q[kKSteps];
  floatx16 acc[kBlocks];
  float m, l;                               // maximum in units of the exponent, the lane's part of the sum

  static __device__ __forceinline__ int column(int lane) { return lane & 31; }
  static __device__ __forceinline__ int k_place(int row, int chunk) { return chunk ^ (row & (kChunks - 1)); }
  static __device__ __forceinline__ int v_place(int row, int chunk) { return chunk ^ (kD == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1)); }
  __device__ __forceinline__ void load_q(const char* row, int lane) {
#pragma unroll
    for (int c = 0; c < kKSteps; ++c) q[c] = *reinterpret_cast<const uintx4*>(row + (2 * c + (lane >> 5)) * 16);
  }
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) acc[e] = floatx16{0};
  }
  // Where a lane reads: chunk 2 c + h of token r is at k_at ^ 32 c, the four rows of v_operand from v_at on.  (Steps start at multiples of 1 KB.)
  static __device__ __forceinline__ uint32_t k_at(int lane) { return (lane & 31) * kRowBytes + k_place(lane & 31, lane >> 5) * 16; }
  static __device__ __forceinline__ uint32_t v_at(int lane) {
    const int i = lane & 15, row = 4 * (lane >> 5) + (i >> 2);
    return row * kRowBytes + v_place(row, 2 * (lane >> 4 & 1) + (i >> 1 & 1)) * 16 + (i & 1) * 8;
  }
  // The operand of tokens 16 u .., dimensions 32 e ..
  static __device__ __forceinline__ bf16x8 v_operand(uint32_t v_lds, int u, int e) {
    bf16x8 f;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const bf16x4 x = lds_turned((v_lds ^ (64 * e)) + (16 * u + 8 * w) * kRowBytes);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * w + j] = x[j];
    }
    return f;
  }
  // Scores; -inf where `seen` says so.  meanwhile(): what is done while the matrix instructions run, and gives `seen`.
  template <class F>
  __device__ __forceinline__ void scores(floatx16& s, uint32_t k_lds, int lane, F meanwhile) const {
    s = floatx16{0};
    uintx4 k[kKSteps];
#pragma unroll
    for (int c = 0; c < kKSteps; ++c) k[c] = lds_chunk(k_lds ^ (32 * c));
    __builtin_amdgcn_sched_barrier(0);          // all of them on their way before the first is waited for
#pragma unroll
    for (int c = 0; c < kKSteps; ++c)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[c]), __builtin_bit_cast(bf16x8, q[c]), s, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    const Seen seen = meanwhile();
    if (seen.masked) {
      asm volatile("");                         // (a branch: few steps go this way, and as selects it is a third of the instructions)
      const uint32_t mine = seen.bits >> (4 * (lane >> 5));
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = mine >> (8 * (i >> 2) + (i & 3)) & 1 ? s[i] : -INFINITY;
    }
  }
  template <class F>
  __device__ __forceinline__ void step(uint32_t k_lds, uint32_t v_lds, float scale, float rise, int lane, F meanwhile) {
    floatx16 s;
    bf16x8 v[2][kBlocks];
    scores(s, k_lds, lane, [&] {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) v[u][e] = v_operand(v_lds, u, e);
      const Seen seen = meanwhile();
      __builtin_amdgcn_sched_barrier(0);
      return seen;
    });
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(pair_max<32>(top) * scale, m);
    if (__ballot(top > m + rise)) {
      const float f = factor_of(m, top);
      m = top;
      l *= f;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) acc[e] *= f;
    }
    const float base = exponent_base(m);
    float sum = 0.f;
    uint32_t hi[8], lo[8];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      float p[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        p[x] = __builtin_amdgcn_exp2f(fmaf(s[i + x], scale, -base));
        sum += p[x];
      }
      const uint32_t b0 = __float_as_uint(p[0]), b1 = __float_as_uint(p[1]);
      hi[i / 2] = __builtin_amdgcn_perm(b1, b0, 0x07060302);
      const bf16x2 rest = {(__bf16)(p[0] - __uint_as_float(b0 & 0xffff0000u)), (__bf16)(p[1] - __uint_as_float(b1 & 0xffff0000u))};
      lo[i / 2] = __builtin_bit_cast(uint32_t, rest);
    }
    l += sum;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8 ph = __builtin_bit_cast(bf16x8, uintx4{hi[4 * u], hi[4 * u + 1], hi[4 * u + 2], hi[4 * u + 3]});
      const bf16x8 pl = __builtin_bit_cast(bf16x8, uintx4{lo[4 * u], lo[4 * u + 1], lo[4 * u + 2], lo[4 * u + 3]});
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) {
        acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[u][e], ph, acc[e], 0, 0, 0);
        acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[u][e], pl, acc[e], 0, 0, 0);
      }
    }
  }
  // Bits of the tokens whose weight is not zero.
  __device__ __forceinline__ uint32_t weighs(uint32_t k_lds, Seen seen, float scale, int lane) const {
    floatx16 s;
    scores(s, k_lds, lane, [&] { return seen; });
    const float base = exponent_base(m);
    uint32_t bits = 0, other, mine;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (__builtin_amdgcn_exp2f(fmaf(s[i], scale, -base)) != 0.f) bits |= 1u << (8 * (i >> 2) + (i & 3));
    lane_pair<32>(bits << (4 * (lane >> 5)), mine, other);
    return mine | other;
  }
  // The values of a token (number `row` in the LDS) that are not finite, with weight `on` (NaN if that is zero).
  __device__ __forceinline__ void add_not_finite(uint32_t v_stage, int row, bool seen, bool on, int lane) {
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int dim = 32 * e + 8 * q4 + 4 * (lane >> 5);
        const uintx4 v = lds_chunk(v_stage + row * kRowBytes + v_place(row, dim / 8) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = lane >> 5 ? v[2 + j / 2] : v[j / 2], x = j & 1 ? w & 0xffff0000u : w << 16;
          if ((x & 0x7f800000u) == 0x7f800000u) acc[e][4 * q4 + j] += seen ? on ? __uint_as_float(x) : NAN : 0.f;
        }
      }
  }
  // A chunk of values without those that are not finite.
  static __device__ __forceinline__ uintx4 finite(uintx4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0x0000ffffu;
      if ((v[i] & 0x00007f80u) == 0x00007f80u) v[i] &= 0xffff0000u;
    }
    return v;
  }
  __device__ __forceinline__ bool any_nan_or_large() const {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = __builtin_elementwise_maximum(x, fabsf(acc[e][i]));
    return __ballot(!(x < kLarge)) != 0;
  }
  __device__ __forceinline__ float whole_sum() const { return pair_sum<32>(l); }
  static __device__ __forceinline__ bool writes_sum(int lane) { return lane < 32; }
  // f(first of four dimensions, their sums) for all that a lane has of its row.
  template <class F>
  __device__ __forceinline__ void each(int lane, F f) const {
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 4) f(32 * e + 2 * i + 4 * (lane >> 5), floatx4{acc[e][i], acc[e][i + 1], acc[e][i + 2], acc[e][i + 3]});
  }
  static constexpr int kQuads = 4 * kBlocks;    // of a lane's sums
  __device__ __forceinline__ floatx4 quad(int i) const { return {acc[i / 4][4 * (i & 3)], acc[i / 4][4 * (i & 3) + 1], acc[i / 4][4 * (i & 3) + 2], acc[i / 4][4 * (i & 3) + 3]}; }
  __device__ __forceinline__ void set_quad(int i, floatx4 x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i / 4][4 * (i & 3) + j] = x[j];
  }
  // The row divided by its sum: lanes h and 32 + h have four dimensions each of the same eight, and exchange them for eight each of sixteen.
  __device__ __forceinline__ void store(char* to, float sum, int lane, bool mine) const {
    const float by = 1.0f / sum;
    const auto part = [&](float o) { return (__bf16)(sum == 0.f ? 0.f : o * by); };
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 8) {
        uintx4 t;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
          const auto pair = [&](int at) { return __builtin_bit_cast(uint32_t, bf16x2{part(acc[e][at]), part(acc[e][at + 1])}); };
          const auto both = __builtin_amdgcn_permlane32_swap(pair(i + 2 * j), pair(i + 4 + 2 * j), false, false);
          t[j] = both[0];
          t[2 + j] = both[1];
        }
        if (mine) *reinterpret_cast<uintx4*>(to + (32 * e + 2 * i + 8 * (lane >> 5)) * 2) = t;
      }
  }
};

// f32: 16 rows, 16x16x4 instructions, 16 tokens.  S^T = K Q^T: lane (g, r) holds chunk 4 c + g of token r, four products; the score is the sum of four sums of d / 4.
// Of the result lane (g, n) holds tokens 4 g + j of row n: the B operand of O^T += V^T P^T for tokens j, 4 + j, 8 + j, 12 + j.  The A operand: lane (g, r)
// holds dimensions 64 x + 4 r .. of token 4 g + j; output block 4 x + y has dimensions 64 x + 4 r + y.
template <int kD>
struct Rows<false, kD> {
  static constexpr int kRows = 16, kTokens = 16, kKSteps = kD / 16, kBlocks = kD / 16, kRowBytes = kD * 4, kChunks = kRowBytes / 16;
  uintx4 q[kKSteps];
  floatx4 acc[kBlocks];
  float m, l;

  static __device__ __forceinline__ int column(int lane) { return lane & 15; }
  static __device__ __forceinline__ int k_place(int row, int chunk) { return chunk ^ (row & 15); }
  static __device__ __forceinline__ int v_place(int row, int chunk) { return chunk; }
  // Chunk 4 c + g of token r is at k_at ^ 64 c, chunk r of token 4 g at v_at.
  static __device__ __forceinline__ uint32_t k_at(int lane) { return (lane & 15) * kRowBytes + k_place(lane & 15, lane >> 4) * 16; }
  static __device__ __forceinline__ uint32_t v_at(int lane) { return 4 * (lane >> 4) * kRowBytes + (lane & 15) * 16; }
  __device__ __forceinline__ void load_q(const char* row, int lane) {
#pragma unroll
    for (int c = 0; c < kKSteps; ++c) q[c] = *reinterpret_cast<const uintx4*>(row + (4 * c + (lane >> 4)) * 16);
  }
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) acc[e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  template <class F>
  __device__ __forceinline__ void scores(floatx4& s, uint32_t k_lds, int lane, F meanwhile) const {
    floatx4 x[4] = {};
    uintx4 k[kKSteps];
#pragma unroll
    for (int c = 0; c < kKSteps; ++c) k[c] = lds_chunk(k_lds ^ (64 * c));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < kKSteps; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[c][e]), __uint_as_float(q[c][e]), x[e], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    const Seen seen = meanwhile();
    s = (x[0] + x[1]) + (x[2] + x[3]);
    if (seen.masked) {
      asm volatile("");
      const uint32_t mine = seen.bits >> (4 * (lane >> 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = mine >> j & 1 ? s[j] : -INFINITY;
    }
  }
  template <class F>
  __device__ __forceinline__ void step(uint32_t k_lds, uint32_t v_lds, float scale, float rise, int lane, F meanwhile) {
    floatx4 s;
    uintx4 v[4][kD / 64];
    scores(s, k_lds, lane, [&] {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < kD / 64; ++x) v[j][x] = lds_chunk(v_lds + j * kRowBytes + 256 * x);
      const Seen seen = meanwhile();
      __builtin_amdgcn_sched_barrier(0);
      return seen;
    });
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    top = fmaxf(pair_max<16>(pair_max<32>(top)) * scale, m);
    if (__ballot(top > m + rise)) {
      const float f = factor_of(m, top);
      m = top;
      l *= f;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) acc[e] *= f;
    }
    const float base = exponent_base(m);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], scale, -base));
      sum += s[j];
    }
    l += sum;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int x = 0; x < kD / 64; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[4 * x + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[j][x][y]), s[j], acc[4 * x + y], 0, 0, 0);
  }
  __device__ __forceinline__ uint32_t weighs(uint32_t k_lds, Seen seen, float scale, int lane) const {
    floatx4 s;
    scores(s, k_lds, lane, [&] { return seen; });
    const float base = exponent_base(m);
    uint32_t bits = 0, x, y;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (__builtin_amdgcn_exp2f(fmaf(s[j], scale, -base)) != 0.f) bits |= 1u << j;
    lane_pair<32>(bits << (4 * (lane >> 4)), x, y);
    lane_pair<16>(x | y, x, y);
    return x | y;
  }
  __device__ __forceinline__ void add_not_finite(uint32_t v_stage, int row, bool seen, bool on, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < kD / 64; ++x) {
        const uintx4 v = lds_chunk(v_stage + row * kRowBytes + 256 * x + (4 * (lane >> 4) + i) * 16);
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if ((v[y] & 0x7f800000u) == 0x7f800000u) acc[4 * x + y][i] += seen ? on ? __uint_as_float(v[y]) : NAN : 0.f;
      }
  }
  static __device__ __forceinline__ uintx4 finite(uintx4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] = 0u;
    return v;
  }
  __device__ __forceinline__ bool any_nan_or_large() const {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) x = __builtin_elementwise_maximum(x, fabsf(acc[e][i]));
    return __ballot(!(x < kLarge)) != 0;
  }
  __device__ __forceinline__ float whole_sum() const { return pair_sum<16>(pair_sum<32>(l)); }
  static __device__ __forceinline__ bool writes_sum(int lane) { return lane < 16; }
  template <class F>
  __device__ __forceinline__ void each(int lane, F f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < kD / 64; ++x)
        f(64 * x + 4 * (4 * (lane >> 4) + i), floatx4{acc[4 * x][i], acc[4 * x + 1][i], acc[4 * x + 2][i], acc[4 * x + 3][i]});
  }
  static constexpr int kQuads = kBlocks;
  __device__ __forceinline__ floatx4 quad(int i) const { return acc[i]; }
  __device__ __forceinline__ void set_quad(int i, floatx4 x) { acc[i] = x; }
  __device__ __forceinline__ void store(char* to, float sum, int lane, bool mine) const {
    each(lane, [&](int dim, floatx4 o) { if (mine) *reinterpret_cast<floatx4*>(to + dim * 4) = normalised(o, sum); });
  }
};

// A workgroup has a wave for every kRows rows of a tile; each takes every token (every second step, where two waves share rows).  Of a ring of kStages steps in the LDS one is worked on, the others are on
// their way there.  A step has 16 KB at d = 128, 8 KB at 64, in either type.  Eight waves have eight steps, one workgroup to a compute unit; four waves 64 KB, two workgroups.  Two waves
// have four steps: 64 KB and two workgroups of cut sequences at d = 128, 32 KB and four workgroups at 64.  Short sequences at d = 128, which are not cut, want
// more workgroups, not more steps ahead: two steps and four workgroups (64 sequences of 60 tokens, bf16: 16.4 -> 12.1 us; 512 of them 110 -> 87, and 77 in a later run).
template <bool kBf16, int kD, int kWaves, bool kSplit>
struct Geometry {
  using R = Rows<kBf16, kD>;
  static constexpr int kThreads = 64 * kWaves, kStep = R::kTokens, kRowTile = R::kRows * kWaves;
  static constexpr int kHalfBytes = kStep * R::kRowBytes, kStageBytes = 2 * kHalfBytes;      // K, then V: 8 or 16 KB
  static constexpr int kLoads = kStageBytes / 1024 / kWaves;                                 // of a wave for a step, 1 KB each
  static constexpr bool kLarge = kStageBytes > 8 * 1024;
  static constexpr int kStages = kWaves == 8 ? 8 : kWaves == 4 ? (kLarge ? 4 : 8) : kLarge && !kSplit ? 2 : 4;
  static constexpr int kGroups = kWaves == 8 ? 1 : kWaves == 4 ? 2 : kLarge && kSplit ? 2 : 4;         // workgroups that a compute unit holds
  static constexpr int kMostWays = kWaves == 8 || kStages < 4 ? 1 : 2;       // steps that waves of the same rows may have side by side
  static constexpr int kStateBytes = R::kQuads * 1024 + 512;   // what a wave hands over
  static constexpr int kWavesPerSimd = (kGroups * kWaves + 3) / 4;
  static constexpr int kPlacesAt = kStages * kStageBytes, kIdsAt = kPlacesAt + 2 * kWindow * 8;       // places of K and V, page ids
  static constexpr int kLiveAt = kIdsAt + 2 * kWindow * 4, kVoteAt = kLiveAt + 2 * kWindow / 8, kLdsBytes = kVoteAt + 16;
  static_assert(kGroups * kLdsBytes <= 160 * 1024, "the LDS");
  static_assert((kWaves - 1) * kStateBytes <= kPlacesAt && (kStages & (kStages - 1)) == 0, "the ring");
};

// All but the youngest `steps` requests of a wave have landed, of kLoads each; more than kMost are not waited for.
template <int kMost, int kLoads>
__device__ __forceinline__ void wait_for_all_but(int steps) {
  if (steps >= kMost) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMost * kLoads) : "memory");
  else if constexpr (kMost > 0) wait_for_all_but<kMost - 1, kLoads>(steps);
}

template <bool kBf16, int kD, int kWaves, bool kSplit>
__global__ __launch_bounds__(64 * kWaves, (Geometry<kBf16, kD, kWaves, kSplit>::kWavesPerSimd)) void tree_kernel(TreeArgs a) {
  using G = Geometry<kBf16, kD, kWaves, kSplit>;
  using R = Rows<kBf16, kD>;
  constexpr int kLead = kSplit ? tree_lead(G::kStep) : 0, kThreads = G::kThreads;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int* const ids = reinterpret_cast<int*>(smem + G::kIdsAt);
  uint2* const places_at = reinterpret_cast<uint2*>(smem + G::kPlacesAt);
  uint64_t* const live_at = reinterpret_cast<uint64_t*>(smem + G::kLiveAt);      // bits of the tokens that there are
  int* const vote = reinterpret_cast<int*>(smem + G::kVoteAt);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto places_of = [&](const Sequence& s) {       // of one unit
    return kSplit ? tree_steps(s.len, G::kStep) + kLead : 1;
  };
  auto all_places = [&](const Sequence& s) { return tree_units(s.n * a.group, G::kRowTile) * places_of(s); };

  // The run of this workgroup, and the head and sequence that its first place is of.  Neighbours on the axis run on one XCD: a KV head, or several, where there are eight or more.
  const int group = (blockIdx.x & 7) * (a.groups >> 3) + (blockIdx.x >> 3);
  int b = 0, first = 0, of_head, run = 1, kvh = 0;        // of_head: places of a head; first: of the sequence, among them all
  Sequence mine_of{};                             // of n <= 64: that of the lane's sequence
  if (a.n <= kPlanBatch) {                        // a few sequences to a lane
    const int each = (a.n + 63) / 64;
    int mine = 0;
    int fewest = 0;
    if (each == 1) {
      if (lane < a.n) {
        mine_of = sequence_of(a, lane);
        mine = all_places(mine_of);
        fewest = mine_of.n;
      }
    } else {                                      // (their lengths asked for at once)
#pragma unroll
      for (int i = 0; i < kPlanBatch / 64; ++i) {
        const int at = lane * each + i;
        const Sequence s = sequence_of(a, min(at, a.n - 1));
        mine += i < each && at < a.n ? all_places(s) : 0;
        fewest = min(fewest, s.n);
      }
    }
    if (__ballot(fewest < 0)) return;
    const int upto = (int)wave_scan((uint32_t)mine, sum_of);
    of_head = __builtin_amdgcn_readlane(upto, 63);
    if (kSplit) run = (of_head * a.heads_kv + a.runs - 1) / a.runs;
    if (group * run >= of_head * a.heads_kv) return;
    kvh = group * run / of_head;
    const int pos = group * run - kvh * of_head, at = __builtin_ctzll(__ballot(upto > pos));
    first = kvh * of_head + __builtin_amdgcn_readlane(upto - mine, at);
    b = at * each;
  } else {                                        // the last sequence that begins at or before the run: 64 candidates at a time
    of_head = a.first_place[a.n];
    if (kSplit) run = (of_head * a.heads_kv + a.runs - 1) / a.runs;
    if (group * run >= of_head * a.heads_kv) return;
    kvh = group * run / of_head;
    for (int n = a.n; n > 1;) {
      const int apart = (n + 63) / 64, at = lane * apart;
      const bool before = at < n && a.first_place[b + min(at, n - 1)] <= group * run - kvh * of_head;
      const int skip = (__builtin_popcountll(__ballot(before)) - 1) * apart;
      b += skip;
      n = min(apart, n - skip);
    }
    first = kvh * of_head + a.first_place[b];
  }
  const int begin = group * run, end = min(begin + run, of_head * a.heads_kv);

  for (int pos = begin; pos < end;) {
    if (b >= a.n) {
      if (++kvh >= a.heads_kv) return;
      b = 0;
    }
    Sequence seq;
    if (a.n <= 64) seq = {__builtin_amdgcn_readlane(mine_of.len, b), __builtin_amdgcn_readlane(mine_of.row0, b), __builtin_amdgcn_readlane(mine_of.n, b)};
    else seq = sequence_of(a, b);
    const int rows = seq.n * a.group, units = tree_units(rows, G::kRowTile), places = places_of(seq);
    if (pos >= first + units * places) {          // (a sequence without rows has no places)
      first += units * places;
      ++b;
      continue;
    }
    const int unit = (pos - first) / places, unit_first = first + unit * places, seq_b = b;
    const int steps = tree_steps(seq.len, G::kStep);
    int t0 = 0, t1 = steps, place = 0, last = 0;
    bool whole = true;
    if constexpr (kSplit) {
      const DecodePiece piece = decode_piece(unit_first, steps, group, run, kLead);
      pos = unit_first + places;
      if (piece.t1 <= piece.t0) continue;         // the run ends before its first step
      whole = piece.t0 == 0 && piece.t1 == steps;
      place = decode_part(piece, group);
      t0 = piece.t0;
      t1 = piece.t1;
      if (t0 == 0 && !whole) last = decode_last_group(unit_first, steps, run, kLead);
    } else {
      pos = end;
    }
    const bool has_first = t0 == 0;               // the unit's first step
    const int base = seq.len - seq.n, unit_rows = min(G::kRowTile, rows - unit * G::kRowTile);
    // no row of a chain sees more than its last one's token
    const int limit = a.masks ? seq.len : max(min(seq.len, base + (int)a.per_token.div(unit * G::kRowTile + unit_rows - 1) + 1), 0);
    t1 = min(t1, (limit + G::kStep - 1) / G::kStep);

    R rw;
    const uint32_t ring = lds_address(smem), k_lane = R::k_at(lane), v_lane = R::v_at(lane);
    // Of few rows half of the waves have no work; they take every second step of the same rows then, two steps to a barrier, and hand their sums over in the end.  A wave alone
    // takes longer for a step than memory does: 16 rows of 16 sequences of 4000, f32, d = 128, 120 -> 99 us; 64 of 32 of 1000 to 16000, bf16, 154 -> 142.  Four steps side by
    // side, of eight waves, are slower (168 and 155 us of 32 to 96 rows): too few are on their way.
    const int needed = unit_rows > 4 * R::kRows ? 8 : unit_rows > 2 * R::kRows ? 4 : unit_rows > R::kRows ? 2 : 1;
    const int way = wave / needed;
    auto attend = [&](auto constant) {
      constexpr int ways = decltype(constant)::value;
      const int row_first = (wave & (needed - 1)) * R::kRows;        // of the unit
      const bool works = row_first < unit_rows && way < ways;
      const int my_row = unit * G::kRowTile + min(row_first + R::column(lane), unit_rows - 1);
      const int my_token = (int)a.per_token.div(my_row), my_head = kvh * a.group + my_row - my_token * a.group;
      const int32_t* const table = a.table + (int64_t)seq_b * a.table_stride;
      const char* const k_head = a.k + kvh * a.k_h;
      const char* const v_head = a.v + kvh * a.v_h;
      // Page ids of a window of tokens, on their way to the LDS like everything else; then their tokens' places.
      auto fetch_ids = [&](int window) {
        const int tok0 = window * kWindow, p0 = (int)a.page.div(min(tok0, limit - 1)), last = (int)a.page.div(limit - 1);
        for (int i = wave; i < kWindow / 64; i += kWaves)
          word_to_lds(table + min(p0 + 64 * i + lane, last), ring + G::kIdsAt + ((window & 1) * kWindow + 64 * i) * 4);
      };
      const int window0 = t0 * G::kStep / kWindow;
      if (t0 < t1) {
        fetch_ids(window0);
        fetch_ids(window0 + 1);
      }
      rw.load_q(a.q + (seq.row0 + my_token) * a.q_t + my_head * a.q_h, lane);
      // the first two words of the row's mask, all of them as a rule
      const uint64_t* const my_mask = a.masks ? a.masks + (seq.row0 + my_token) * a.mask_stride : nullptr;
      const uint64_t mask0 = a.masks ? my_mask[0] : 0, mask1 = a.masks && a.words > 1 ? my_mask[1] : 0;
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0f70);           // vmcnt(0), for the compiler to know: it would wait for the queries in the loop, and for the ring with them
      auto place_tokens = [&](int window) {         // everyone is there before and after
        const int side = window & 1, tok0 = window * kWindow, p0 = (int)a.page.div(tok0);
#pragma unroll
        for (int at = tid; at < kWindow; at += kThreads) {
          const int tok = min(tok0 + at, limit - 1), p = (int)a.page.div(tok), off = tok - p * (int)a.page.d;      // (behind the last: that one's place again)
          const uint32_t id = ids[side * kWindow + p - p0];
          const bool held = id < (uint32_t)a.pages;
          places_at[side * kWindow + at] = held ? make_uint2(id * a.k_b + off * a.k_l, id * a.v_b + off * a.v_l) : make_uint2(0u, 0u);
          const uint64_t live = __ballot(held && tok0 + at < limit);
          if (lane == 0) live_at[(side * kWindow + at) >> 6] = live;
        }
      };
      // What a lane fetches of a step: 16 bytes of K or V of a token in each of its wave's requests.
      const char* from[G::kLoads];
      int from_row[G::kLoads];
      bool from_v[G::kLoads];
#pragma unroll
      for (int i = 0; i < G::kLoads; ++i) {
        const int chunk = i * kWaves + wave, in_half = chunk % (G::kHalfBytes / 1024), c = lane % R::kChunks;
        from_row[i] = in_half * (1024 / R::kRowBytes) + lane / R::kChunks;
        from_v[i] = chunk >= G::kHalfBytes / 1024;
        from[i] = from_v[i] ? v_head + R::v_place(from_row[i], c) * 16 : k_head + R::k_place(from_row[i], c) * 16;
      }
      auto issue = [&](int step, int stage) {
#pragma unroll
        for (int i = 0; i < G::kLoads; ++i) {
          const uint2 at = places_at[(step * G::kStep + from_row[i]) & (2 * kWindow - 1)];
          to_lds(from[i] + ((uint64_t)(from_v[i] ? at.y : at.x) << a.unit), ring + stage * G::kStageBytes + (i * kWaves + wave) * 1024);
        }
      };
      // Steps in turn, `ways` at a time: body(the first, next), which has everyone call next() once.
      auto stage_of = [&](int step) { return ring + ((step - t0) & (G::kStages - 1)) * G::kStageBytes; };
      bool again = false;
      auto traverse = [&](auto body) {
        int placed = window0;                       // the last window whose tokens' places are there
        if (t0 < t1) {
          if (again) {
            fetch_ids(placed);
            fetch_ids(placed + 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          }
          again = true;
          meet();
          place_tokens(placed);
          meet();
        }
        auto request = [&](int step) {              // (uniform, and so are the barriers in it)
          if (step >= t1) return;
          if (step * G::kStep / kWindow != placed) {        // its ids were asked for a window ago, and have landed with the step that everyone has waited for
            ++placed;
            place_tokens(placed);
            meet();
            fetch_ids(placed + 1);
          }
          issue(step, (step - t0) & (G::kStages - 1));
        };
        static_assert(kWindow / G::kStep >= G::kStages, "page ids that have landed, places that no one reads any more");
#pragma clang loop unroll(disable)
        for (int i = 0; i < G::kStages - ways; ++i) request(t0 + i);
#pragma clang loop unroll(disable)
        for (int t = t0; t < t1; t += ways) {
          // all but my youngest requests have landed; after the barrier everyone's have, and everyone is done with the steps before
          wait_for_all_but<G::kStages - 2, G::kLoads>(min(G::kStages - 2 * ways, max(t1 - ways - t, 0)));
          meet();
          body(t, [&] {
#pragma clang loop unroll(disable)
            for (int i = 0; i < ways; ++i) request(t + G::kStages - ways + i);
          });
        }
        meet();
      };
      auto seen_of = [&](int t) {                   // of the wave's tokens: whether there are any that the lane's row does not see, and which it does
        const int tok0 = t * G::kStep, at = tok0 - base;         // `at`: of the first token among the new ones
        constexpr uint32_t kAll = ~0u >> (32 - G::kStep);
        const uint32_t live = __builtin_amdgcn_readfirstlane(reinterpret_cast<const uint32_t*>(live_at)[(tok0 & (2 * kWindow - 1)) >> 5] >> (tok0 & 31)) & kAll;
        Seen s{at > -G::kStep || live != kAll, kAll};
        if (s.masked) {
          s.bits = chain_bits(my_token, at);
          if (my_mask) {
            const int w = max(at, 0) >> 6;
            if (w == 0) s.bits = tree_bits(mask0, mask1, at);
            else s.bits = tree_bits(w == 1 ? mask1 : w < a.words ? my_mask[w] : 0, w + 1 < a.words ? my_mask[w + 1] : 0, at);
          }
          s.bits &= live;
        }
        return s;
      };
      // Once as it is.  A weight of zero, or a part of one that is, times infinity or NaN is NaN, also where a row does not see the token: if there is NaN, or a sum that is
      // too large, in the result of a workgroup, once more with the values that are finite and with weights up to 1, and then the others added to the rows that see them.
      bool clean = false;
#pragma clang loop unroll(disable)
      for (;;) {
        rw.clear();
        traverse([&](int t, auto next) {
          if (clean) {
            for (int step = t; step < min(t + ways, t1); ++step)
              for (int i = tid; i < G::kHalfBytes / 16; i += kThreads) {
                const lds_chunk_ptr_t at = (lds_chunk_ptr_t)(uintptr_t)(stage_of(step) + G::kHalfBytes + i * 16);
                *at = R::finite(*at);
              }
            meet();
          }
          if (!works || t + way >= t1) {
            next();
            return;
          }
          const uint32_t stage = stage_of(t + way);
          rw.step(stage + k_lane, stage + G::kHalfBytes + v_lane, a.scale_log2e, clean ? 0.f : kRise, lane, [&] {
            const Seen seen = seen_of(t + way);
            next();
            return seen;
          });
        });
        if (clean) break;
        if (tid == 0) *vote = 0;
        meet();
        if (works && rw.any_nan_or_large() && lane == 0) *vote = 1;
        meet();
        if (!*vote) break;
        clean = true;
      }
      if (clean) {
        traverse([&](int t, auto next) {
          next();
          if (!works || t + way >= t1) return;
          const Seen seen = seen_of(t + way);
          const uint32_t stage = stage_of(t + way), on = rw.weighs(stage + k_lane, seen, a.scale_log2e, lane);
#pragma clang loop unroll(disable)
          for (int i = 0; i < G::kStep; ++i) rw.add_not_finite(stage + G::kHalfBytes, i, seen.bits >> i & 1, on >> i & 1, lane);
        });
      }
      if constexpr (ways > 1) {                     // the ring is free
        auto state_of = [&](int from) { return smem + (from - needed) * G::kStateBytes; };
        if (works && way > 0) {
          char* const to = state_of(wave);
#pragma unroll
          for (int i = 0; i < R::kQuads; ++i) *reinterpret_cast<floatx4*>(to + (i * 64 + lane) * 16) = rw.quad(i);
          *reinterpret_cast<float2*>(to + R::kQuads * 1024 + lane * 8) = make_float2(rw.m, rw.l);
        }
        meet();
        if (works && way == 0)
#pragma clang loop unroll(disable)
          for (int w = 1; w < ways; ++w) {
            const char* const from = state_of(wave + w * needed);
            const float2 ml = *reinterpret_cast<const float2*>(from + R::kQuads * 1024 + lane * 8);
            const float top = fmaxf(rw.m, ml.x), f = factor_of(rw.m, top), x = factor_of(ml.x, top);
            rw.m = top;
            rw.l = rw.l * f + ml.y * x;
#pragma unroll
            for (int i = 0; i < R::kQuads; ++i) rw.set_quad(i, rw.quad(i) * f + *reinterpret_cast<const floatx4*>(from + (i * 64 + lane) * 16) * x);
          }
      }

      float sum = rw.whole_sum();
      // The row of a new token that has no slot is that of a query without any token: of a sequence that was not served the last tokens are none of the new ones.  (Asked for
      // here: in front of the loop it would take a register in it.)
      if (a.slots && (uint64_t)a.slots[seq.row0 + my_token] >= (uint64_t)a.all_slots) {
        rw.m = -INFINITY;
        sum = 0.f;
      }
      const int row = row_first + R::column(lane);  // of the unit
      const bool there = row < unit_rows && way == 0;
      const int64_t id = (int64_t)(seq.row0 + my_token) * a.heads_kv * a.group + my_head;
      if (kSplit && has_first && there && R::writes_sum(lane)) a.cut_of[id] = whole ? -1 : pack_cut(group, last, row);
      if (whole) {
        rw.store(a.out + (seq.row0 + my_token) * a.out_t + my_head * a.out_h, sum, lane, there);
        if (a.lse && there && R::writes_sum(lane)) a.lse[id] = lse_of(rw.m, sum);
      } else if (there) {
        const int64_t to = (int64_t)place * G::kRowTile + row;
        rw.each(lane, [&](int dim, floatx4 o) { *reinterpret_cast<floatx4*>(a.part_o + to * kD + dim) = o; });
        if (R::writes_sum(lane)) a.part_ml[to] = make_float2(rw.m, sum);
      }
    };
    const int most_ways = min(kWaves / needed, G::kMostWays);     // (constants, for the loops of one step at a time: 3% of large trees)
    if (most_ways <= 1) attend(std::integral_constant<int, 1>{});
    else if constexpr (G::kMostWays > 1) attend(std::integral_constant<int, 2>{});
    if constexpr (kSplit) meet();
  }
}

// First places of many sequences: one workgroup, a run of sequences to a thread.  (Up to kPlanBatch a launch less: 64 sequences 12.1 us in all.)
__global__ __launch_bounds__(1024) void tree_plan_kernel(TreeArgs a, int step, int tile, bool split) {
  __shared__ int wave_sum[16], wave_falls[16];
  const int tid = threadIdx.x, each = (a.n + 1023) / 1024, i0 = min(tid * each, a.n), i1 = min(i0 + each, a.n);
  bool falls = false;
  auto places = [&](int i) {
    const Sequence s = sequence_of(a, i);
    falls |= s.n < 0;
    return tree_units(s.n * a.group, tile) * (split ? tree_steps(s.len, step) + tree_lead(step) : 1);
  };
  int mine = 0;
  for (int i = i0; i < i1; ++i) mine += places(i);
  const int upto = (int)wave_scan((uint32_t)mine, sum_of);
  const bool any_falls = __ballot(falls) != 0;
  if ((tid & 63) == 63) {
    wave_sum[tid >> 6] = upto;
    wave_falls[tid >> 6] = any_falls;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = upto - mine, fall = 0;
  for (int w = 0; w < tid >> 6; ++w) at += wave_sum[w];
  for (int w = 0; w < 16; ++w) fall |= wave_falls[w];
  for (int i = i0; i < i1; ++i) {
    a.first_place[i] = at;
    at += places(i);
  }
  if (tid == 1023) a.first_place[a.n] = fall ? 0 : at;
}

// The pieces of a row that more than one workgroup had a part in, added up, a wave to a row: 4 numbers to a lane, a part to every d / 4 lanes, four of them asked for at once.  In the
// order of heads that the runs have, so that a row is added up where its parts were made, whose L2 has them: one sequence of 700 tokens, 22 parts to a row, 9.7 us in the order of
// rows, 5.6 in this.
constexpr int kJoinThreads = 256;
template <bool kBf16, int kD>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(TreeArgs a, int tile, int groups) {
  constexpr int kLanes = kD / 4, kSubs = 64 / kLanes, kRows = kJoinThreads / 64, kElem = kBf16 ? 2 : 4, kParts = 4;
  const int lane = threadIdx.x & 63, c = lane % kLanes, rows = a.tokens * a.group, of_head = (rows + kRows - 1) / kRows;
  const int group = (blockIdx.x & 7) * (groups >> 3) + (blockIdx.x >> 3), kvh = group / of_head, r = (group - kvh * of_head) * kRows + (threadIdx.x >> 6);
  if (kvh >= a.heads_kv || r >= rows) return;
  const int t = (int)a.per_token.div(r), head = kvh * a.group + r - t * a.group;
  const int64_t id = (int64_t)t * a.heads_kv * a.group + head;
  const int cut = a.cut_of[id], begin = a.cu[0], end = a.cu[a.n];
  const int g0 = cut & (kMostRuns - 1), g1 = min(cut / kMostRuns & (kMostRuns - 1), a.runs - 1), row = cut / (kMostRuns * kMostRuns);
  if (cut < 0 || t < begin || t >= end || row >= tile) return;       // (a row of no sequence has anything there)
  float m = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int w0 = g0 + lane / kLanes; w0 <= g1; w0 += kSubs * kParts) {
    float2 ml[kParts];
    floatx4 p[kParts];
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      // place 1 of the run that it begins in, place 0 of the others
      const int w = min(w0 + j * kSubs, g1);
      const int64_t place = (int64_t)(2 * w + (w == g0)) * tile + row;
      ml[j] = a.part_ml[place];
      p[j] = *reinterpret_cast<const floatx4*>(a.part_o + place * kD + 4 * c);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kParts; ++j) top = fmaxf(top, ml[j].x);
    const float old = factor_of(m, top);
    m = top;
    l *= old;
    o *= old;
#pragma unroll
    for (int j = 0; j < kParts; ++j) {
      if (w0 + j * kSubs > g1) break;
      const float f = factor_of(ml[j].x, top);
      l = fmaf(ml[j].y, f, l);
      o += p[j] * f;
    }
  }
#pragma unroll
  for (int off = kLanes; off < 64; off *= 2) {
    const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), top = fmaxf(m, m2), f = factor_of(m, top), x = factor_of(m2, top);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * f + __shfl_xor(o[i], off) * x;
    m = top;
    l = l * f + l2 * x;
  }
  o = normalised(o, l);
  // Parts that are numbers and a sum that is none: every part by its share of the whole sum.
  const float most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(o[0]), fabsf(o[1])), __builtin_elementwise_maximum(fabsf(o[2]), fabsf(o[3])));
  if (__ballot(!(most < INFINITY))) {
    const float by = 1.0f / l;
    o = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int w = g0 + lane / kLanes; w <= g1; w += kSubs) {
      const int64_t place = (int64_t)(2 * w + (w == g0)) * tile + row;
      o += *reinterpret_cast<const floatx4*>(a.part_o + place * kD + 4 * c) * factor_of(a.part_ml[place].x, m) * by;
    }
#pragma unroll
    for (int off = kLanes; off < 64; off *= 2)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], off);
  }
  if (lane >= kLanes) return;
  store4<kBf16>(a.out + t * a.out_t + head * a.out_h + c * 4 * kElem, o);
  if (a.lse && c == 0) a.lse[id] = lse_of(m, l);
}

// Waves of a workgroup, rows of its tile, tokens of a step, workgroups that the device holds: by the rows that a sequence has on average.
struct Variant { int waves, tile, step, runs; };
template <bool kBf16, int kD, int kWaves>
constexpr Variant variant() {
  using G = Geometry<kBf16, kD, kWaves, true>;
  return {kWaves, G::kRowTile, G::kStep, 256 * G::kGroups};
}
// f(bf16, d, waves) of a call as constants
template <class F>
auto with_waves(bool bf16, int d, int waves, F f) {
  auto pick = [&](auto w) {
    if (bf16) return d == 128 ? f(std::true_type{}, std::integral_constant<int, 128>{}, w) : f(std::true_type{}, std::integral_constant<int, 64>{}, w);
    return d == 128 ? f(std::false_type{}, std::integral_constant<int, 128>{}, w) : f(std::false_type{}, std::integral_constant<int, 64>{}, w);
  };
  return waves == 2 ? pick(std::integral_constant<int, 2>{}) : waves == 4 ? pick(std::integral_constant<int, 4>{}) : pick(std::integral_constant<int, 8>{});
}
// Short sequences are not cut: a workgroup for a unit, and no join.  Of 64 / 8 sequences (8 KV heads, 8 new tokens), not cut and cut: bf16, d = 128, 500 tokens 43 / 20 us
// and 33 / 16, 120 tokens 14 / 10.5 and 18 / 10.5; d = 64, 490 tokens 20.8 / 17.1 and 28.1 / 13.6; f32, d = 64, 230 tokens 32 / 18.5 and 37 / 15, d = 128, 110 tokens 45 / 19 and 30 / 15.
bool is_solo(int row_tokens, int d, bool bf16) { return (int64_t)row_tokens * d <= (bf16 ? 32768 : 8192); }
// Two waves where they have all of the rows, and where more workgroups to a compute unit can be had for it: f32, d = 128, 16 sequences of 4000, 32 rows 142 us, and 166 of four
// waves; but bf16 at d = 128 124 us of 4 rows, and 117 of four waves, whose ring is as large and is filled by more.  Four or eight: the fewer rows that
// the last tile leaves empty.  Of 128 rows (bf16, d = 128, 32 sequences of 1000 to 16000) 193 us with four waves, 227 with eight; of 192 290 with either; of 288 469 and 482, but of
// 640 850 and 819, 1152 1506 and 1405: bf16 takes four for up to three tiles only.  f32 (16 sequences of 2000): 144 rows 252 and 320, 320 436 and 483, 832 1152 and 1190.
constexpr int least_waves(bool bf16, int d, bool split) { return bf16 && d == 128 && split ? 4 : 2; }
Variant variant_of(int tokens, int n, int group, int d, bool bf16, int row_tokens) {
  const int64_t wave_rows = bf16 ? 32 : 16, rows = ((int64_t)tokens * group + n - 1) / n;
  const int least = least_waves(bf16, d, !is_solo(row_tokens, d, bf16));
  return with_waves(bf16, d, rows <= 2 * wave_rows ? least : (!bf16 || rows <= 12 * wave_rows) && align_up(rows, 8 * wave_rows) > align_up(rows, 4 * wave_rows) ? 4 : 8, [](auto b, auto d, auto w) {
    return variant<decltype(b)::value, decltype(d)::value, decltype(w)::value>();
  });
}
int64_t most_units(int tokens, int n, int heads_kv, int group, int tile) {
  return heads_kv * ((int64_t)tokens * group / tile + std::min(n, tokens));
}
int64_t most_places(int tokens, int n, int heads_kv, int group, const Variant& v, int row_tokens) {
  return most_units(tokens, n, heads_kv, group, v.tile) * (tree_steps(row_tokens, v.step) + tree_lead(v.step));
}
struct TreeWs { size_t first_place, cut_of, part_o, part_ml, total; };
TreeWs carve(int n, int64_t rows, int64_t runs, int tile, int d) {
  TreeWs w;
  size_t o = 0;
  w.first_place = o; o += align_up((size_t)(n + 1) * 4, 256);
  w.cut_of = o; o += align_up((size_t)(runs ? rows : 0) * 4, 256);
  w.part_o = o; o += align_up((size_t)2 * runs * tile * d * 4, 256);
  w.part_ml = o; o += align_up((size_t)2 * runs * tile * 8, 256);
  w.total = o;
  return w;
}

template <bool kBf16, int kD, int kWaves, bool kSplit>
basa_status launch_kernel(const TreeArgs& a, hipStream_t st) {
  using G = Geometry<kBf16, kD, kWaves, kSplit>;
  const auto kernel = tree_kernel<kBf16, kD, kWaves, kSplit>;
  if (a.n > kPlanBatch) {
    ProfScope prof(K_TREE, st);
    tree_plan_kernel<<<1, 1024, 0, st>>>(a, G::kStep, G::kRowTile, kSplit);
    BASA_HIP_CHECK_LAUNCH("tree_plan_kernel");
  }
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
  if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(dynamic LDS)");
  ProfScope prof(K_TREE, st);
  kernel<<<a.groups, G::kThreads, G::kLdsBytes, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("tree_kernel");
  return BASA_OK;
}
template <bool kBf16, int kD, int kWaves>
basa_status launch(const TreeArgs& a, bool solo, hipStream_t st) {
  using G = Geometry<kBf16, kD, kWaves, true>;
  if (solo) return launch_kernel<kBf16, kD, kWaves, false>(a, st);
  basa_status s = BASA_OK;
  if constexpr (kWaves >= least_waves(kBf16, kD, true)) s = launch_kernel<kBf16, kD, kWaves, true>(a, st);
  if (s != BASA_OK) return s;
  ProfScope prof(K_TREE_JOIN, st);
  static_assert(256 * G::kGroups <= kMostRuns && G::kRowTile <= kMostRows, "a packed cut");
  constexpr int kRows = kJoinThreads / 64;
  const int groups = (int)align_up((size_t)a.heads_kv * ceil_div(a.tokens * a.group, kRows), 8);
  tree_join_kernel<kBf16, kD><<<groups, kJoinThreads, 0, st>>>(a, G::kRowTile, groups);
  BASA_HIP_CHECK_LAUNCH("tree_join_kernel");
  return BASA_OK;
}

}  // namespace

bool tree_takes(int tokens, int n, int heads_q, int heads_kv, int d, bool bf16, int row_tokens) {
  const int group = heads_q / heads_kv;
  return n == 0 || most_places(tokens, n, heads_kv, group, variant_of(tokens, n, group, d, bf16, row_tokens), row_tokens) < INT_MAX / 2;
}
size_t tree_workspace_bytes(int tokens, int n, int heads_q, int heads_kv, int d, bool bf16, int row_tokens) {
  if (n == 0) return 256;
  const int group = heads_q / heads_kv;
  const Variant v = variant_of(tokens, n, group, d, bf16, row_tokens);
  if (is_solo(row_tokens, d, bf16)) return carve(n, 0, 0, 0, 0).total;
  return carve(n, (int64_t)tokens * heads_q, std::min<int64_t>(v.runs, most_places(tokens, n, heads_kv, group, v, row_tokens)), v.tile, d).total;
}

// Tokens' places are 32-bit numbers, in units of the largest power of two up to 256 that divides the strides of pages and tokens, in bytes: 16 at least, and
// a row in all stores of whole rows.  -1: K or V reaches further than those numbers do.
int tree_place_unit(const TensorView& k, const TensorView& v) {
  const int64_t e = k.dtype == BASA_BF16 ? 2 : 4;
  int unit = 8;
  for (const TensorView* t : {&k, &v})
    for (int64_t stride : {t->stride_b, t->stride_l})
      while ((stride * e) & ((1 << unit) - 1)) --unit;
  for (const TensorView* t : {&k, &v}) {
    const double reach = ((double)(t->batch - 1) * t->stride_b + (double)(t->L - 1) * t->stride_l) * e;
    if (reach >= 4294967295.0 * (1 << unit)) return -1;
  }
  return unit;
}

basa_status launch_tree_attn(const TensorView& q, const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width,
                             int64_t table_stride, const int32_t* lens, const int32_t* cu, int n, const int64_t* masks, int words,
                             int64_t mask_stride, const int64_t* slots, void* out, int64_t out_st, int64_t out_sh, float* lse, void* ws, hipStream_t st) {
  if (n == 0) return BASA_OK;
  TreeArgs a{};
  const bool bf16 = q.dtype == BASA_BF16;
  const int e = bf16 ? 2 : 4;
  a.q = static_cast<const char*>(q.ptr); a.k = static_cast<const char*>(k_pages.ptr); a.v = static_cast<const char*>(v_pages.ptr);
  a.q_t = q.stride_l * e; a.q_h = q.stride_h * e;
  a.k_h = k_pages.stride_h * e; a.v_h = v_pages.stride_h * e;
  a.unit = tree_place_unit(k_pages, v_pages);
  auto in_units = [&](int64_t stride) { return (uint32_t)(stride * e >> a.unit); };
  a.k_b = in_units(k_pages.stride_b); a.k_l = in_units(k_pages.stride_l); a.v_b = in_units(v_pages.stride_b); a.v_l = in_units(v_pages.stride_l);
  a.table = table; a.table_stride = table_stride; a.lens = lens; a.cu = cu;
  a.n = n; a.tokens = q.L; a.heads_kv = k_pages.heads; a.group = q.heads / k_pages.heads; a.pages = k_pages.batch;
  a.row_tokens = width * k_pages.L;
  a.page = fast_div((uint32_t)k_pages.L);
  a.per_token = fast_div((uint32_t)a.group);
  a.slots = slots; a.all_slots = (int64_t)k_pages.batch * k_pages.L;
  a.masks = reinterpret_cast<const uint64_t*>(masks); a.words = words; a.mask_stride = mask_stride;
  a.out = static_cast<char*>(out); a.out_t = out_st * e; a.out_h = out_sh * e; a.lse = lse;
  const Variant v = variant_of(a.tokens, n, a.group, q.d, bf16, a.row_tokens);
  const int64_t units = most_units(a.tokens, n, a.heads_kv, a.group, v.tile);
  const bool solo = is_solo(a.row_tokens, q.d, bf16);
  a.runs = solo ? 0 : (int)std::min<int64_t>(v.runs, most_places(a.tokens, n, a.heads_kv, a.group, v, a.row_tokens));
  a.groups = (int)align_up(solo ? units : a.runs, 8);
  const TreeWs w = carve(n, (int64_t)q.L * q.heads, a.runs, v.tile, q.d);
  char* base = static_cast<char*>(ws);
  a.first_place = reinterpret_cast<int*>(base + w.first_place);
  a.cut_of = reinterpret_cast<int*>(base + w.cut_of);
  a.part_o = reinterpret_cast<float*>(base + w.part_o);
  a.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)q.d);
  return with_waves(bf16, q.d, v.waves, [&](auto b, auto d, auto w) {
    return launch<decltype(b)::value, decltype(d)::value, decltype(w)::value>(a, solo, st);
  });
}

}  // namespace basa
