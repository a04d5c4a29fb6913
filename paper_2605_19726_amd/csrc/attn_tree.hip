// Attention of several new tokens of every sequence, a tree or a chain of drafted ones, over its pages of the key-value cache (gfx950).
//
// A sequence holds `len` tokens, of which the last n are the new ones (their rows of q; keys and values are in the pages); base = len - n.  Token t sees
// every token before base, and new token j if bit j of its mask is set (a chain: j <= t).  Rows of a KV head: (t, h), n x group of them.  For
// a row:  s_j = q . k_j,  m = max s_j,  o = sum_j e^((s_j - m) / sqrt(d)) v_j / sum_j e^((s_j - m) / sqrt(d)),  lse = m / sqrt(d) + ln sum, over the tokens
// that it sees.  One pass over the tokens with a running maximum and sum per row.
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
typedef const __attribute__((address_space(3))) uintx4* lds_chunk_ptr_t;
typedef __attribute__((address_space(3))) short4v* lds_quad_ptr_t;

struct TreeArgs {
  const char *q, *k, *v;
  int64_t q_t, q_h;                         // strides in bytes
  int64_t k_h, v_h;
  uint32_t k_b, k_l, v_b, v_l;              // of a page and of a token, in units of 16 bytes
  const int32_t *table, *lens, *cu;
  int64_t table_stride;
  int n, tokens, heads_kv, group, pages;    // sequences; rows of q
  int row_tokens;                           // tokens a table row has room for
  FastDiv page, per_token;                  // per_token: division by the group
  const uint64_t* masks;                    // or null: chains
  int64_t mask_stride;
  int words;
  char* out;
  int64_t out_t, out_h;                     // in bytes
  float* lse;                               // [tokens][heads_q] or null
  int groups;                               // workgroups, a multiple of 8
  int runs;                                 // at most so many runs (cut by runs)
  int* first_place;                         // workspace: [n + 1] first place of every sequence, then how many there are
  float* part_o;                            // [2 runs][tile][d], not normalised
  float2* part_ml;                          // [2 runs][tile] maximum in units of the exponent, sum
  float scale_log2e;                        // log2 e / sqrt(d)
};
__device__ const uint4 kZeroRow[32] = {};   // the row of a token whose page is none

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 32;                   // tokens that a wave takes at a time
constexpr int kPlanBatch = 512;             // up to this many sequences every wave sums up the lengths by itself
constexpr int kWindow = 1024, kWindowPages = kWindow + 4;     // tokens whose page ids are in the LDS, twice

struct Sequence { int len, row0, n; };
__device__ __forceinline__ Sequence sequence_of(const TreeArgs& a, int b) {
  Sequence s;
  s.len = min(max(a.lens[b], 0), a.row_tokens);
  s.row0 = min(max(a.cu[b], 0), a.tokens);
  s.n = max(min(a.cu[b + 1], a.tokens) - s.row0, 0);
  return s;
}
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
// p times this lies 3/4 to 3/2 steps of bf16 below p, so that its rounding is below p and the rest is positive.
constexpr float kBelow = 1.f - 0x3p-9f;

// 16 bytes from memory for every lane, side by side into the LDS.  Written in assembly, without a register for its result: the compiler would wait for all of
// these before it reads the LDS or meets a barrier; the waits stand where the ring needs them.
template <bool kOnce>
__device__ __forceinline__ void to_lds(const char* from, uint32_t at) {
  if constexpr (kOnce) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "s"(at) : "memory");
  else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "memory");
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

// What a wave does with 32 tokens in the LDS for its rows.  Row of a lane: its column of the matrix instruction.
template <bool kBf16, int kD> struct Rows;

// bf16: 32 rows, 32x32x16 instructions.  S^T = K Q^T: lane (h, r) of the A operand holds chunk 2 c + h of token r at step c.  Of the result lane (h, n) holds
// tokens 8 q + 4 h + j (register 4 q + j) of row n: the B operand of O^T += V^T P^T for tokens 16 u .. 16 u + 15, if token 16 u + 8 w + 4 h + j stands at place
// 8 h + 4 w + j of the sum.  The A operand in that order: the transposing read gives lane i of 16 column i of the four rows that they address.
template <int kD>
struct Rows<true, kD> {
  static constexpr int kRows = 32, kKSteps = kD / 16, kBlocks = kD / 32, kRowBytes = kD * 2, kChunks = kRowBytes / 16;
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
  // The operand of tokens 16 u .. of the wave's 32, dimensions 32 e ..
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
  // kMasked: `seen` has a bit for every token that the lane's row sees.  kSafe: see below.
  template <bool kMasked, bool kSafe>
  __device__ __forceinline__ void step(uint32_t k_lds, uint32_t v_lds, uint32_t seen, float scale, int lane) {
    const int h = lane >> 5;
    floatx16 s = floatx16{0};
#pragma unroll
    for (int c = 0; c < kKSteps; ++c)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, lds_chunk(k_lds ^ (32 * c))), __builtin_bit_cast(bf16x8, q[c]), s, 0, 0, 0);
    if constexpr (kMasked) {
      const uint32_t mine = seen >> (4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = mine >> (8 * (i >> 2) + (i & 3)) & 1 ? s[i] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(pair_max<32>(top) * scale, m);
    if (__ballot(top != m)) {
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
      float p[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        p[x] = __builtin_amdgcn_exp2f(fmaf(s[i + x], scale, -base));
        sum += p[x];
      }
      uint32_t b0, b1;
      if constexpr (kSafe) {
        b0 = __float_as_uint((float)(__bf16)(p[0] * kBelow));
        b1 = __float_as_uint((float)(__bf16)(p[1] * kBelow));
      } else {
        b0 = __float_as_uint(p[0]) & 0xffff0000u;
        b1 = __float_as_uint(p[1]) & 0xffff0000u;
      }
      hi[i / 2] = __builtin_amdgcn_perm(b1, b0, 0x07060302);
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 rest = {(__bf16)(p[0] - __uint_as_float(b0)), (__bf16)(p[1] - __uint_as_float(b1))};
      lo[i / 2] = __builtin_bit_cast(uint32_t, rest);
    }
    l += sum;
    bf16x8 ph[2], pl[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ph[u] = __builtin_bit_cast(bf16x8, uintx4{hi[4 * u], hi[4 * u + 1], hi[4 * u + 2], hi[4 * u + 3]});
      pl[u] = __builtin_bit_cast(bf16x8, uintx4{lo[4 * u], lo[4 * u + 1], lo[4 * u + 2], lo[4 * u + 3]});
    }
    if constexpr (kMasked && kSafe) {
      // token by token, added where it is seen: what a row does not see may be anything
#pragma unroll
      for (int e = 0; e < kBlocks; ++e)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 v = v_operand(v_lds, u, e);
#pragma clang loop unroll(disable)
          for (int t = 0; t < 16; ++t) {
            bf16x8 one;
#pragma unroll
            for (int i = 0; i < 8; ++i) one[i] = t == 8 * (i >> 2) + 4 * h + (i & 3) ? v[i] : (__bf16)0.f;
            floatx16 x = floatx16{0};
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, ph[u], x, 0, 0, 0);
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, pl[u], x, 0, 0, 0);
            const bool on = seen >> (16 * u + t) & 1;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[e][i] = on ? acc[e][i] + x[i] : acc[e][i];
          }
        }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) {
          const bf16x8 v = v_operand(v_lds, u, e);
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, ph[u], acc[e], 0, 0, 0);
          acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pl[u], acc[e], 0, 0, 0);
        }
    }
  }
  __device__ __forceinline__ bool any_nan() const {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = __builtin_elementwise_maximum(x, acc[e][i]);
    return __ballot(x != x) != 0;
  }
  __device__ __forceinline__ float whole_sum() const { return pair_sum<32>(l); }
  static __device__ __forceinline__ bool writes_sum(int lane) { return lane < 32; }
  template <int kPitch>
  __device__ __forceinline__ void store(float* part, int lane) const {       // to row column(lane) of `part`
    float* row = part + (lane & 31) * kPitch + 4 * (lane >> 5);
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<floatx4*>(row + 32 * e + 8 * q4) = floatx4{acc[e][4 * q4], acc[e][4 * q4 + 1], acc[e][4 * q4 + 2], acc[e][4 * q4 + 3]};
  }
};

// f32: 16 rows, 16x16x4 instructions, the tokens in two halves of 16.  S^T = K Q^T: lane (g, r) holds chunk 4 c + g of token r, four products; the score is the sum
// of four sums of d / 4.  Of the result lane (g, n) holds tokens 4 g + j of row n: the B operand of O^T += V^T P^T for tokens j, 4 + j, 8 + j, 12 + j.  The A
// operand: lane (g, r) holds dimensions 64 x + 4 r .. of token 4 g + j; output block 4 x + y has dimensions 64 x + 4 r + y.
template <int kD>
struct Rows<false, kD> {
  static constexpr int kRows = 16, kKSteps = kD / 16, kBlocks = kD / 16, kRowBytes = kD * 4, kChunks = kRowBytes / 16;
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
  template <bool kMasked, bool kSafe>
  __device__ __forceinline__ void step(uint32_t k_lds, uint32_t v_lds, uint32_t seen, float scale, int lane) {
    const int g = lane >> 4;
    floatx4 s[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      floatx4 x[4] = {};
#pragma unroll
      for (int c = 0; c < kKSteps; ++c) {
        const uintx4 k = lds_chunk((k_lds ^ (64 * c)) + 16 * half * kRowBytes);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), x[e], 0, 0, 0);
      }
      s[half] = (x[0] + x[1]) + (x[2] + x[3]);
      if constexpr (kMasked) {
        const uint32_t mine = seen >> (16 * half + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[half][j] = mine >> j & 1 ? s[half][j] : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, s[half][j]);
    top = fmaxf(pair_max<16>(pair_max<32>(top)) * scale, m);
    if (__ballot(top != m)) {
      const float f = factor_of(m, top);
      m = top;
      l *= f;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) acc[e] *= f;
    }
    const float base = exponent_base(m);
    float sum = 0.f;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[half][j] = __builtin_amdgcn_exp2f(fmaf(s[half][j], scale, -base));
        sum += s[half][j];
      }
    l += sum;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < kD / 64; ++x) {
          const uintx4 v = lds_chunk(v_lds + (16 * half + j) * kRowBytes + 256 * x);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            floatx4& o = acc[4 * x + y];
            if constexpr (kMasked && kSafe) {
#pragma clang loop unroll(disable)
              for (int t = 0; t < 4; ++t) {
                const floatx4 one = __builtin_amdgcn_mfma_f32_16x16x4f32(t == g ? __uint_as_float(v[y]) : 0.f, s[half][j], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                const bool on = seen >> (16 * half + 4 * t + j) & 1;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = on ? o[i] + one[i] : o[i];
              }
            } else {
              o = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[y]), s[half][j], o, 0, 0, 0);
            }
          }
        }
  }
  __device__ __forceinline__ bool any_nan() const {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) x = __builtin_elementwise_maximum(x, acc[e][i]);
    return __ballot(x != x) != 0;
  }
  __device__ __forceinline__ float whole_sum() const { return pair_sum<16>(pair_sum<32>(l)); }
  static __device__ __forceinline__ bool writes_sum(int lane) { return lane < 16; }
  template <int kPitch>
  __device__ __forceinline__ void store(float* part, int lane) const {
    float* row = part + (lane & 15) * kPitch;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < kD / 64; ++x)
        *reinterpret_cast<floatx4*>(row + 64 * x + 4 * (4 * (lane >> 4) + i)) = floatx4{acc[4 * x][i], acc[4 * x + 1][i], acc[4 * x + 2][i], acc[4 * x + 3][i]};
  }
};

// kRowWaves waves side by side over the rows of a tile, the others over the tokens of a step.  Of a ring of kStages steps in the LDS one is worked on, the
// others are on their way there.
template <bool kBf16, int kD, int kRowWaves>
struct Geometry {
  using R = Rows<kBf16, kD>;
  static constexpr int kTokenWaves = kWaves / kRowWaves, kStep = kTile * kTokenWaves, kRowTile = R::kRows * kRowWaves;
  static constexpr int kHalfBytes = kStep * R::kRowBytes, kStageBytes = 2 * kHalfBytes;      // K, then V
  static constexpr int kLoads = kHalfBytes / 1024 / kWaves;                                  // per wave, of K and of V each
  static constexpr int kStages = kStageBytes >= 64 * 1024 ? 2 : kStageBytes >= 32 * 1024 ? 2 : 4;
  static constexpr int kPitch = kD + 4;
  static constexpr int kPartBytes = kWaves * R::kRows * kPitch * 4;
  static constexpr int kIdsAt = kStages * kStageBytes;
  static constexpr int kRingBytes = kIdsAt + 2 * kWindowPages * 4;
  static constexpr int kMlAt = (kRingBytes > kPartBytes ? kRingBytes : kPartBytes) / 16 * 16 + 16;
  static constexpr int kLdsBytes = kMlAt + kWaves * R::kRows * 8 + 16;       // then the vote, and whether a window has pages that are none
  static constexpr int kGroups = kLdsBytes > 80 * 1024 ? 1 : 2;                // workgroups that a compute unit holds
};

template <bool kBf16, int kD, int kRowWaves, bool kSplit, bool kOnce>
__global__ __launch_bounds__(kThreads, (Geometry<kBf16, kD, kRowWaves>::kGroups)) void tree_kernel(TreeArgs a) {
  using G = Geometry<kBf16, kD, kRowWaves>;
  using R = Rows<kBf16, kD>;
  constexpr int kElem = kBf16 ? 2 : 4, kLead = kSplit ? tree_lead(G::kStep) : 0;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int* const ids = reinterpret_cast<int*>(smem + G::kIdsAt);
  float* const part = reinterpret_cast<float*>(smem);
  float2* const part_ml = reinterpret_cast<float2*>(smem + G::kMlAt);
  int* const vote = reinterpret_cast<int*>(smem + G::kMlAt + kWaves * R::kRows * 8);
  int* const holes = vote + 1;                    // [2]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row_wave = wave % kRowWaves, token_wave = wave / kRowWaves;
  auto places_of = [&](const Sequence& s) {       // of one unit
    return kSplit ? tree_steps(s.len, G::kStep) + kLead : 1;
  };
  auto all_places = [&](const Sequence& s) { return tree_units(s.n * a.group, G::kRowTile) * places_of(s) * a.heads_kv; };

  // the run of this workgroup and the sequence that its first place is of.  Neighbours on the axis run on one XCD
  const int group = (blockIdx.x & 7) * (a.groups >> 3) + (blockIdx.x >> 3);
  int b = 0, first = 0, total, run = 1;
  if (a.n <= kPlanBatch) {                        // a few sequences to a lane
    const int each = (a.n + 63) / 64;
    int mine = 0;
    for (int i = 0; i < each; ++i) {
      const int at = lane * each + i;
      if (at < a.n) mine += all_places(sequence_of(a, at));
    }
    const int upto = (int)wave_scan((uint32_t)mine, sum_of);
    total = __builtin_amdgcn_readlane(upto, 63);
    if constexpr (kSplit) run = (total + a.runs - 1) / a.runs;
    if (group * run >= total) return;
    const int at = __builtin_ctzll(__ballot(upto > group * run));
    first = __builtin_amdgcn_readlane(upto - mine, at);
    b = at * each;
    if (kSplit && group == 0 && tid == 0) a.first_place[a.n] = total;
  } else {                                        // the last sequence that begins at or before the run: 64 candidates at a time
    total = a.first_place[a.n];
    if constexpr (kSplit) run = (total + a.runs - 1) / a.runs;
    if (group * run >= total) return;
    for (int n = a.n; n > 1;) {
      const int apart = (n + 63) / 64, at = lane * apart;
      const bool before = at < n && a.first_place[b + min(at, n - 1)] <= group * run;
      const int skip = (__builtin_popcountll(__ballot(before)) - 1) * apart;
      b += skip;
      n = min(apart, n - skip);
    }
    first = a.first_place[b];
  }
  const int begin = group * run, end = min(begin + run, total);

  for (int pos = begin; pos < end && b < a.n;) {    // (offsets that do not ascend may have places for no one)
    const Sequence seq = sequence_of(a, b);
    const int rows = seq.n * a.group, units = tree_units(rows, G::kRowTile), places = places_of(seq);
    if (pos >= first + units * places * a.heads_kv) {        // (a sequence without rows has no places)
      first += units * places * a.heads_kv;
      ++b;
      continue;
    }
    const int index = (pos - first) / places, unit_first = first + index * places;
    const int kvh = index / units, unit = index - kvh * units, seq_b = b;
    int t0 = 0, t1 = tree_steps(seq.len, G::kStep), place = 0;
    bool whole = true;
    if constexpr (kSplit) {
      const DecodePiece piece = decode_piece(unit_first, t1, group, run, kLead);
      pos = unit_first + places;
      if (piece.t1 <= piece.t0) continue;         // the run ends before its first step
      whole = piece.t0 == 0 && piece.t1 == t1;
      place = decode_part(piece, group);
      t0 = piece.t0;
      t1 = piece.t1;
      if (a.n <= kPlanBatch && index == 0 && t0 == 0 && tid == 0) a.first_place[seq_b] = first;
    } else {
      pos = end;
    }
    const int base = seq.len - seq.n, unit_rows = min(G::kRowTile, rows - unit * G::kRowTile);
    // no row of a chain sees more than its last one's token
    const int limit = a.masks ? seq.len : max(min(seq.len, base + (int)a.per_token.div(unit * G::kRowTile + unit_rows - 1) + 1), 0);
    t1 = min(t1, (limit + G::kStep - 1) / G::kStep);

    R rw;
    const uint32_t ring = lds_address(smem), k_lane = R::k_at(lane), v_lane = R::v_at(lane);
    const int row_first = row_wave * R::kRows;    // of the unit
    const bool works = row_first < unit_rows;
    const int my_row = unit * G::kRowTile + min(row_first + R::column(lane), unit_rows - 1);
    const int my_token = (int)a.per_token.div(my_row), my_head = kvh * a.group + my_row - my_token * a.group;
    rw.load_q(a.q + (seq.row0 + my_token) * a.q_t + my_head * a.q_h, lane);
    __builtin_amdgcn_s_waitcnt(0x0f70);           // vmcnt(0), for the compiler to know: it would wait for the queries in the loop, and for the ring with them
    const uint64_t* const my_mask = a.masks ? a.masks + (seq.row0 + my_token) * a.mask_stride : nullptr;

    const int32_t* const table = a.table + (int64_t)seq_b * a.table_stride;
    const char* const k_head = a.k + kvh * a.k_h;
    const char* const v_head = a.v + kvh * a.v_h;
    auto fill = [&](int window) {                 // page ids of a window of tokens; everyone is there before and after
      const int tok0 = window * kWindow, side = window & 1;
      if (tid == 0) holes[side] = 0;
      meet();
      const int p0 = (int)a.page.div(tok0), p1 = (int)a.page.div(min(tok0 + kWindow, limit) - 1);
      for (int i = tid; i <= p1 - p0; i += kThreads) {
        const int id = table[p0 + i];
        ids[side * kWindowPages + i] = id;
        if ((unsigned)id >= (unsigned)a.pages) holes[side] = 1;
      }
      meet();
    };
    auto page_of = [&](int tok, int* off) {       // of tokens before `limit`: the id may be that of no page
      const int p = (int)a.page.div(tok), p0 = (int)a.page.div(tok & ~(kWindow - 1));
      *off = tok - p * (int)a.page.d;
      return ids[((tok / kWindow) & 1) * kWindowPages + p - p0];
    };
    auto issue = [&](int step, int stage) {
#pragma unroll
      for (int i = 0; i < G::kLoads; ++i) {
        const int chunk = i * kWaves + wave, row = chunk * (1024 / R::kRowBytes) + lane / R::kChunks, c = lane % R::kChunks;
        int off;
        const int tok = step * G::kStep + row, id = page_of(min(tok, limit - 1), &off);
        const bool valid = (unsigned)id < (unsigned)a.pages && tok < limit;
        const uint64_t k_at = valid ? (uint64_t)(uint32_t)id * a.k_b + (uint64_t)(uint32_t)off * a.k_l : 0;
        const uint64_t v_at = (uint64_t)(uint32_t)id * a.v_b + (uint64_t)(uint32_t)off * a.v_l;
        const char* const k_row = k_head + (k_at << 4);
        const char* const v_row = valid ? v_head + (v_at << 4) : reinterpret_cast<const char*>(kZeroRow);
        const uint32_t to = ring + stage * G::kStageBytes + chunk * 1024;
        to_lds<kOnce>(k_row + R::k_place(row, c) * 16, to);
        to_lds<kOnce>(v_row + R::v_place(row, c) * 16, to + G::kHalfBytes);
      }
    };
    auto pass = [&](auto safe) {
      rw.clear();
      int filled = t0 * G::kStep / kWindow - 1;   // the last window whose page ids are there
      int stage_to = 0, stage_at = 0;
      auto request = [&](int step) {              // (uniform, and so are the barriers in it)
        if (step >= t1) return;
        if (step * G::kStep / kWindow != filled) fill(++filled);
        issue(step, stage_to);
        stage_to = stage_to + 1 == G::kStages ? 0 : stage_to + 1;
      };
#pragma clang loop unroll(disable)
      for (int i = 0; i < G::kStages - 1; ++i) request(t0 + i);
#pragma clang loop unroll(disable)
      for (int t = t0; t < t1; ++t) {
        // all but my youngest requests have landed; after the barrier everyone's have, and everyone is done with the step before
        static_assert(G::kStages == 2 || G::kStages == 4, "these waits");
        if (G::kStages == 2 || t + 1 == t1) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (t + 2 == t1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * G::kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * G::kLoads) : "memory");
        meet();
        request(t + G::kStages - 1);
        const uint32_t k_lds = ring + stage_at * G::kStageBytes + token_wave * kTile * R::kRowBytes, v_lds = k_lds + G::kHalfBytes;
        stage_at = stage_at + 1 == G::kStages ? 0 : stage_at + 1;
        if (!works) continue;
        const int tok0 = t * G::kStep + token_wave * kTile, at = tok0 - base;      // `at`: of the first token among the new ones
        const int hole = __builtin_amdgcn_readfirstlane(holes[t * G::kStep / kWindow & 1]);
        if (at <= -kTile && tok0 + kTile <= limit && !hole) {
          rw.template step<false, decltype(safe)::value>(k_lds + k_lane, v_lds + v_lane, 0u, a.scale_log2e, lane);
        } else {
          int off;
          const int tok = tok0 + (lane & 31), id = page_of(min(tok, limit - 1), &off);
          const uint32_t live = (uint32_t)__ballot(tok < limit && (unsigned)id < (unsigned)a.pages);
          uint32_t seen = chain_bits(my_token, at);
          if (my_mask) {
            const int w = max(at, 0) >> 6;
            seen = tree_bits(w < a.words ? my_mask[w] : 0, w + 1 < a.words ? my_mask[w + 1] : 0, at);
          }
          rw.template step<true, decltype(safe)::value>(k_lds + k_lane, v_lds + v_lane, seen & live, a.scale_log2e, lane);
        }
      }
      meet();
    };
    pass(std::false_type{});
    // A part of a weight may be zero, which times an infinite value is NaN, and so may be the weight of a token that a row does not see.  Nothing else can
    // come of that: a workgroup whose result holds NaN takes its tokens once more, with two positive numbers for every positive weight and the tokens that some row
    // does not see one by one.
    if (tid == 0) *vote = 0;
    meet();
    if (works && rw.any_nan() && lane == 0) *vote = 1;
    meet();
    if (*vote) pass(std::true_type{});

    // the waves that took other tokens of the same rows together
    rw.template store<G::kPitch>(part + wave * R::kRows * G::kPitch, lane);
    const float sum_l = rw.whole_sum();
    if (R::writes_sum(lane)) part_ml[wave * R::kRows + R::column(lane)] = make_float2(rw.m, sum_l);
    meet();
    for (int i = tid; i < unit_rows * (kD / 4); i += kThreads) {
      const int row = i / (kD / 4), c = i % (kD / 4);
      const int at = row;                         // row wave row / kRows, column row % kRows: as they are
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < G::kTokenWaves; ++w) top = fmaxf(top, part_ml[w * G::kRowTile + at].x);
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < G::kTokenWaves; ++w) {
        const float2 ml = part_ml[w * G::kRowTile + at];
        const float f = factor_of(ml.x, top);
        sum = fmaf(ml.y, f, sum);
        o += *reinterpret_cast<const floatx4*>(part + (w * G::kRowTile + at) * G::kPitch + 4 * c) * f;
      }
      if (whole) {
        const int r = unit * G::kRowTile + row, t = (int)a.per_token.div(r), head = kvh * a.group + r - t * a.group;
        store4<kBf16>(a.out + (seq.row0 + t) * a.out_t + head * a.out_h + c * 4 * kElem, normalised(o, sum));
        if (a.lse && c == 0) a.lse[(int64_t)(seq.row0 + t) * a.heads_kv * a.group + head] = lse_of(top, sum);
      } else {
        const int64_t to = (int64_t)place * G::kRowTile + row;
        *reinterpret_cast<floatx4*>(a.part_o + to * kD + 4 * c) = o;
        if (c == 0) a.part_ml[to] = make_float2(top, sum);
      }
    }
    if constexpr (kSplit) meet();
  }
}

// First places of many sequences: one workgroup, a run of sequences to a thread.
__global__ __launch_bounds__(1024) void tree_plan_kernel(TreeArgs a, int step, int tile, bool split) {
  __shared__ int wave_sum[16];
  const int tid = threadIdx.x, each = (a.n + 1023) / 1024, i0 = min(tid * each, a.n), i1 = min(i0 + each, a.n);
  auto places = [&](int i) {
    const Sequence s = sequence_of(a, i);
    return tree_units(s.n * a.group, tile) * (split ? tree_steps(s.len, step) + tree_lead(step) : 1) * a.heads_kv;
  };
  int mine = 0;
  for (int i = i0; i < i1; ++i) mine += places(i);
  const int upto = (int)wave_scan((uint32_t)mine, sum_of);
  if ((tid & 63) == 63) wave_sum[tid >> 6] = upto;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = upto - mine;
  for (int w = 0; w < tid >> 6; ++w) at += wave_sum[w];
  for (int i = i0; i < i1; ++i) {
    a.first_place[i] = at;
    at += places(i);
  }
  if (tid == 1023) a.first_place[a.n] = at;
}

// The pieces of a row that more than one workgroup had a part in, added up: 4 numbers to a lane, a part to every d / 4 lanes.
template <bool kBf16, int kD>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a, int step, int tile) {
  constexpr int kLanes = kD / 4, kParts = 64 / kLanes, kElem = kBf16 ? 2 : 4;
  const int lane = threadIdx.x & 63, heads_q = a.heads_kv * a.group;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (int64_t)a.tokens * heads_q) return;
  const int t = (int)(id / heads_q), head = (int)(id - (int64_t)t * heads_q);
  if (t < a.cu[0] || t >= a.cu[a.n]) return;
  int b = 0;                                  // the last sequence that begins at or before the row
  for (int n = a.n; n > 1;) {
    const int apart = (n + 63) / 64, at = lane * apart;
    const bool before = at < n && a.cu[b + min(at, n - 1)] <= t;
    const int skip = max((int)__builtin_popcountll(__ballot(before)) - 1, 0) * apart;
    b += skip;
    n = min(apart, n - skip);
  }
  const Sequence s = sequence_of(a, b);
  if (t < s.row0 || t >= s.row0 + s.n) return;
  const int lead = tree_lead(step), steps = tree_steps(s.len, step), total = a.first_place[a.n], run = (total + a.runs - 1) / a.runs;
  const int kvh = head / a.group, r = (t - s.row0) * a.group + head - kvh * a.group, unit = r / tile, row = r - unit * tile;
  const int first = a.first_place[b] + (kvh * tree_units(s.n * a.group, tile) + unit) * (steps + lead);
  const int g0 = decode_first_group(first, run, lead), g1 = decode_last_group(first, steps, run, lead);
  if (g0 == g1 || g0 < 0 || g1 >= a.runs) return;      // (whole; or offsets that do not ascend)
  const int c = lane % kLanes;
  float m = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int w = g0 + lane / kLanes; w <= g1; w += kParts) {
    const int64_t place = (int64_t)decode_part(decode_piece(first, steps, w, run, lead), w) * tile + row;
    const float2 ml = a.part_ml[place];
    const floatx4 p = *reinterpret_cast<const floatx4*>(a.part_o + place * kD + 4 * c);
    const float top = fmaxf(m, ml.x), f = factor_of(m, top), x = factor_of(ml.x, top);
    m = top;
    l = l * f + ml.y * x;
    o = o * f + p * x;
  }
#pragma unroll
  for (int off = kLanes; off < 64; off *= 2) {
    const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), top = fmaxf(m, m2), f = factor_of(m, top), x = factor_of(m2, top);
    floatx4 o2;
#pragma unroll
    for (int i = 0; i < 4; ++i) o2[i] = __shfl_xor(o[i], off);
    m = top;
    l = l * f + l2 * x;
    o = o * f + o2 * x;
  }
  if (lane >= kLanes) return;
  store4<kBf16>(a.out + t * a.out_t + head * a.out_h + c * 4 * kElem, normalised(o, l));
  if (a.lse && c == 0) a.lse[id] = lse_of(m, l);
}

constexpr int kRuns = 512;
struct Variant { int row_waves, tile, step; };
// By the rows that a sequence has on average: a wave's rows, twice or four times as many.
Variant variant_of(int tokens, int n, int group, int d, bool bf16) {
  const int wave_rows = bf16 ? 32 : 16, least = !bf16 && d == 128 ? 2 : 1;     // (of whose rows two steps for four waves do not fit the LDS)
  const int64_t rows = ((int64_t)tokens * group + n - 1) / n;
  const int row_waves = std::max(rows <= wave_rows ? 1 : rows <= 2 * wave_rows ? 2 : 4, least);
  return {row_waves, row_waves * wave_rows, kTile * (kWaves / row_waves)};
}
int64_t most_units(int tokens, int n, int heads_kv, int group, int tile) {
  return heads_kv * ((int64_t)tokens * group / tile + std::min(n, tokens));
}
int64_t most_places(int tokens, int n, int heads_kv, int group, const Variant& v, int row_tokens) {
  return most_units(tokens, n, heads_kv, group, v.tile) * (tree_steps(row_tokens, v.step) + tree_lead(v.step));
}
bool is_solo(int64_t units, int row_tokens) { return row_tokens <= 512; }
struct TreeWs { size_t first_place, part_o, part_ml, total; };
TreeWs carve(int n, int64_t runs, int tile, int d) {
  TreeWs w;
  size_t o = 0;
  w.first_place = o; o += align_up((size_t)(n + 1) * 4, 256);
  w.part_o = o; o += align_up((size_t)2 * runs * tile * d * 4, 256);
  w.part_ml = o; o += align_up((size_t)2 * runs * tile * 8, 256);
  w.total = o;
  return w;
}

template <bool kBf16, int kD, int kRowWaves, bool kSplit>
basa_status launch_kernel(const TreeArgs& a, hipStream_t st) {
  using G = Geometry<kBf16, kD, kRowWaves>;
  const auto kernel = tree_kernel<kBf16, kD, kRowWaves, kSplit, kRowWaves < 4>;
  if (a.n > kPlanBatch) {
    ProfScope prof(K_TREE, st);
    tree_plan_kernel<<<1, 1024, 0, st>>>(a, G::kStep, G::kRowTile, kSplit);
    BASA_HIP_CHECK_LAUNCH("tree_plan_kernel");
  }
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
  if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(dynamic LDS)");
  ProfScope prof(K_TREE, st);
  kernel<<<a.groups, kThreads, G::kLdsBytes, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("tree_kernel");
  return BASA_OK;
}
template <bool kBf16, int kD, int kRowWaves>
basa_status launch(const TreeArgs& a, bool solo, hipStream_t st) {
  using G = Geometry<kBf16, kD, kRowWaves>;
  if (solo) return launch_kernel<kBf16, kD, kRowWaves, false>(a, st);
  const basa_status s = launch_kernel<kBf16, kD, kRowWaves, true>(a, st);
  if (s != BASA_OK) return s;
  ProfScope prof(K_TREE_JOIN, st);
  const int64_t rows = (int64_t)a.tokens * a.heads_kv * a.group;
  tree_join_kernel<kBf16, kD><<<(int)((rows + 3) / 4), 256, 0, st>>>(a, G::kStep, G::kRowTile);
  BASA_HIP_CHECK_LAUNCH("tree_join_kernel");
  return BASA_OK;
}

}  // namespace

bool tree_takes(int tokens, int n, int heads_q, int heads_kv, int d, bool bf16, int row_tokens) {
  const int group = heads_q / heads_kv;
  return n == 0 || most_places(tokens, n, heads_kv, group, variant_of(tokens, n, group, d, bf16), row_tokens) < INT_MAX / 2;
}
size_t tree_workspace_bytes(int tokens, int n, int heads_q, int heads_kv, int d, bool bf16, int row_tokens) {
  if (n == 0) return 256;
  const int group = heads_q / heads_kv;
  const Variant v = variant_of(tokens, n, group, d, bf16);
  if (is_solo(most_units(tokens, n, heads_kv, group, v.tile), row_tokens)) return carve(n, 0, 0, 0).total;
  return carve(n, std::min<int64_t>(kRuns, most_places(tokens, n, heads_kv, group, v, row_tokens)), v.tile, d).total;
}

basa_status launch_tree_attn(const TensorView& q, const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width,
                             int64_t table_stride, const int32_t* lens, const int32_t* cu, int n, const int64_t* masks, int words,
                             int64_t mask_stride, void* out, int64_t out_st, int64_t out_sh, float* lse, void* ws, hipStream_t st) {
  if (n == 0) return BASA_OK;
  TreeArgs a{};
  const bool bf16 = q.dtype == BASA_BF16;
  const int e = bf16 ? 2 : 4;
  a.q = static_cast<const char*>(q.ptr); a.k = static_cast<const char*>(k_pages.ptr); a.v = static_cast<const char*>(v_pages.ptr);
  a.q_t = q.stride_l * e; a.q_h = q.stride_h * e;
  a.k_h = k_pages.stride_h * e; a.v_h = v_pages.stride_h * e;
  auto chunks = [&](int64_t stride) { return (uint32_t)(stride * e / 16); };
  a.k_b = chunks(k_pages.stride_b); a.k_l = chunks(k_pages.stride_l); a.v_b = chunks(v_pages.stride_b); a.v_l = chunks(v_pages.stride_l);
  a.table = table; a.table_stride = table_stride; a.lens = lens; a.cu = cu;
  a.n = n; a.tokens = q.L; a.heads_kv = k_pages.heads; a.group = q.heads / k_pages.heads; a.pages = k_pages.batch;
  a.row_tokens = width * k_pages.L;
  a.page = fast_div((uint32_t)k_pages.L);
  a.per_token = fast_div((uint32_t)a.group);
  a.masks = reinterpret_cast<const uint64_t*>(masks); a.words = words; a.mask_stride = mask_stride;
  a.out = static_cast<char*>(out); a.out_t = out_st * e; a.out_h = out_sh * e; a.lse = lse;
  const Variant v = variant_of(a.tokens, n, a.group, q.d, bf16);
  const int64_t units = most_units(a.tokens, n, a.heads_kv, a.group, v.tile);
  const bool solo = is_solo(units, a.row_tokens);
  a.runs = solo ? 0 : (int)std::min<int64_t>(kRuns, most_places(a.tokens, n, a.heads_kv, a.group, v, a.row_tokens));
  a.groups = (int)align_up(solo ? units : a.runs, 8);
  const TreeWs w = carve(n, a.runs, v.tile, q.d);
  char* base = static_cast<char*>(ws);
  a.first_place = reinterpret_cast<int*>(base + w.first_place);
  a.part_o = reinterpret_cast<float*>(base + w.part_o);
  a.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)q.d);
  auto pick = [&](auto row_waves) {
    constexpr int W = decltype(row_waves)::value;
    if (bf16) return q.d == 128 ? launch<true, 128, W>(a, solo, st) : launch<true, 64, W>(a, solo, st);
    if constexpr (W > 1) {
      if (q.d == 128) return launch<false, 128, W>(a, solo, st);
    }
    return launch<false, 64, W>(a, solo, st);
  };
  if (v.row_waves == 1) return pick(std::integral_constant<int, 1>{});
  if (v.row_waves == 2) return pick(std::integral_constant<int, 2>{});
  return pick(std::integral_constant<int, 4>{});
}

}  // namespace basa
