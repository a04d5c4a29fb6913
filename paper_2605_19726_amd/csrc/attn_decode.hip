// Attention of one new token of every sequence over its pages of the key-value cache (gfx950).
//
// For a sequence of n cached tokens and a query head h of KV head h / group:  s_j = q . k_j,  m = max_j s_j,
// o = sum_j e^((s_j - m) / sqrt(d)) v_j / sum_j e^((s_j - m) / sqrt(d)),  lse = m / sqrt(d) + ln sum.  One pass over the cache with a
// running maximum and sum per query head.  4 group flops for 2 bytes of bf16: bound by the memory up to a group of several hundred, so that
// everything serves the loads: the matrix instruction takes the query heads of a KV head as its 16 columns, used or not.
//
// Operands straight from memory, no LDS in between.  A wave takes 32 tokens at a time, in two halves of 16.  S^T = K Q^T: lane (g, r) of the
// A operand holds 16 bytes of token r, chunk 4 c + g of its row at step c; the queries are laid out alike.  Loaded like that an instruction
// would take half a line of 128 bytes from each of 16 rows; so two steps are loaded together, whole lines of 8 rows by each
// instruction, and lanes r and r ^ 8 exchange one of their two chunks in registers.  Of the result, lane (g, n) holds tokens
// 4 g .. 4 g + 3 of each half for query head n: as they are, the B operand of O^T += V^T P^T, if token order within the sum is that
// of lane group g: its own eight tokens.  The A operand is eight tokens of one dimension: lane (g, r) loads its group's eight
// tokens, chunk r of each row (whole rows, 16 lanes of 16 bytes), and turns its 8 x 8 block in registers, a byte permutation for two
// numbers; output block e holds dimensions 8 r + e.  The running maximum is that of the lane's own column in every lane.
// bf16: P goes in as the sum of two bf16 numbers (16 bits; the second product is free beside the loads), accumulation and softmax state in
// fp32.  The second number may be zero or negative, which times an infinite value is NaN where p v is infinite.  Nothing else can come of
// that: a wave whose result holds NaN takes its tiles once more with two positive numbers for every positive p (2^-15 p at worst
// in place of 2^-17 p), and the others pay one look at their result.  f32: the same on the fp32 matrix instruction, without the turning.
//
// The work is cut by tokens, not by sequences: paged_plan.hpp.  Every workgroup finds its run in the running sum of the lengths (they are
// on the device), and the pieces that are not a whole sequence are joined by a second kernel.
//
// Measured (a pass that only reads: 7.05 TB/s): 64 sequences of 8000 to 60000 tokens, 32 heads on 8, d = 128, bf16, 7.6 GB: 1170 us a call, with
// the join, 6.5 TB/s (main kernel alone, when it was built: half lines and ordinary loads 1435, whole lines 1330, whole lines and streaming loads
// 1190).  One sequence of 128K: 84 - 87 + 4.5 - 5.4 us; f32, 16 heads of 64, 21 sequences of 3 to 5000: 34 - 35 + 4.1 - 4.6.  Level: the next tile's
// rows asked for before this one's products, 8 waves to a workgroup, fewer instructions in the exchange and in the rescaling.
#include <algorithm>
#include <climits>
#include "common.hpp"
#include "paged_plan.hpp"

namespace basa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));

struct DecodeArgs {
  const char *q, *k, *v;
  int64_t q_b, q_h;                         // strides in bytes
  int64_t k_b, k_h, k_l, v_b, v_h, v_l;
  const int32_t *table, *lens;
  int64_t table_stride;
  int batch, heads_kv, group, units, pages; // units: runs of 16 kNT query heads that share a KV head
  int row_tokens;                           // tokens a table row has room for
  FastDiv page;
  char* out;
  int64_t out_b, out_h;                     // in bytes
  float* lse;                               // [batch][heads_q] or null
  int* first_place;                         // workspace: [batch + 1] first place of every sequence, then how many there are
  int part_heads;                           // query heads of a partial result
  float* part_o;                            // [2 groups][part_heads][d], not normalised
  float2* part_ml;                          // [2 groups][part_heads] maximum, sum
  float scale, scale_log2e;                 // 1 / sqrt(d), log2 e / sqrt(d)
};

// Up to this many sequences every wave sums up the lengths by itself; of more, a kernel in front does.  By itself -> in front, 8 heads on 1: 500
// sequences of 1 to 1100 tokens 22 us, 600 21.4 -> 4.2 + 19.9, 1000 of 1500 148 -> 4.0 + 139, 4000 of 1 to 2000 163 -> 4.3 + 120.
constexpr int kPlanBatch = 512;
__device__ __forceinline__ int cached_tokens(const DecodeArgs& a, int b) { return min(max(a.lens[b], 0), a.row_tokens); }
__device__ __forceinline__ int sum_of(int x, int y) { return x + y; }
__device__ __forceinline__ float column_max(float v) {      // over the four lane groups
  uint32_t x, y;
  lane_pair<32>(__float_as_uint(v), x, y);
  v = fmaxf(__uint_as_float(x), __uint_as_float(y));
  lane_pair<16>(__float_as_uint(v), x, y);
  return fmaxf(__uint_as_float(x), __uint_as_float(y));
}
__device__ __forceinline__ float column_sum(float v) {
  uint32_t x, y;
  lane_pair<32>(__float_as_uint(v), x, y);
  v = __uint_as_float(x) + __uint_as_float(y);
  lane_pair<16>(__float_as_uint(v), x, y);
  return __uint_as_float(x) + __uint_as_float(y);
}
// e^((s - m) / sqrt(d)) with m = -inf where nothing was seen yet
__device__ __forceinline__ float weight_of(float s, float m, float scale_log2e) {
  return __builtin_amdgcn_exp2f((s - (m == -INFINITY ? 0.f : m)) * scale_log2e);
}
__device__ __forceinline__ float lse_of(float m, float l, float scale) {
  return l == 0.f ? -INFINITY : fmaf(m, scale, __logf(l));
}
// p times this lies 3/4 to 3/2 steps of bf16 below p, so that its rounding is below p and the rest is positive, between 2^-10 p and 2^-6 p: a
// bf16 number too down to p = 2^-125.
constexpr float kBelow = 1.f - 0x3p-9f;
// A cache that is read once: its lines are the first to leave the L2.  (Pays only where an instruction takes whole lines of 128 bytes: with half
// lines, whose other half is asked for by the next instruction, they leave before that.)  Not where several units read the same rows.
template <class T, bool kOnce>
__device__ __forceinline__ T load_rows(const char* at) {
  if constexpr (kOnce) return __builtin_nontemporal_load(reinterpret_cast<const T*>(at));
  return *reinterpret_cast<const T*>(at);
}
// Without any weight: zero, whatever the values are.
__device__ __forceinline__ floatx4 normalised(floatx4 o, float sum) {
  return sum == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / sum);
}
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

// kSplit: the cut by runs.  Otherwise a workgroup per (sequence, run of query heads).  kOnce: rows are read by one unit.
template <bool kBf16, int kD, int kNT, int kWaves, bool kSplit, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, 2) void decode_kernel(DecodeArgs a) {
  constexpr int kHeads = 16 * kNT, kElem = kBf16 ? 2 : 4, kThreads = 64 * kWaves;
  constexpr int kKSteps = kD * kElem / 64;               // 16-byte chunks of a K row per lane
  constexpr int kBlocks = kD / 16;                       // output blocks of 16 dimensions
  constexpr int kVLoads = kBf16 ? 1 : kD / 64;           // loads of a V row per lane: kD / 16 numbers (bf16), 4 at a time (f32)
  constexpr int kPitch = kD + 4;
  extern __shared__ __attribute__((aligned(16))) float part[];        // [kWaves][part_heads][kPitch], then their maxima and sums
  __shared__ int64_t row_at[kWaves][2][kDecodeTile];         // K, V
  float2* const part_ml = reinterpret_cast<float2*>(part + kWaves * a.part_heads * kPitch);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, r = lane & 15;
  const int per_seq = a.heads_kv;

  // the run of this workgroup (or its sequence and head) and the sequence that its first place is of: every wave finds them for itself
  int b = 0, first = 0, run = 0, begin = 0, end = 1, group = blockIdx.x, sub = 0;
  if (a.units > 1) {                            // those of the units of one run: at the same time on one XCD, whose L2 has the rows then
    const int line = blockIdx.x / (8 * a.units), rest = blockIdx.x - line * 8 * a.units;
    group = line * 8 + (rest & 7);
    sub = rest >> 3;
  }
  if constexpr (kSplit) {
    if (a.batch <= kPlanBatch) {                // a few sequences to a lane
      const int each = (a.batch + 63) / 64;
      int places[kPlanBatch / 64], mine = 0;
#pragma unroll
      for (int i = 0; i < kPlanBatch / 64; ++i) {
        const int at = lane * each + i, n = decode_places(cached_tokens(a, min(at, a.batch - 1)));
        places[i] = i < each && at < a.batch ? n : 0;
        mine += places[i];
      }
      const int upto = (int)wave_scan((uint32_t)mine, sum_of), total = __builtin_amdgcn_readlane(upto, 63) * per_seq;
      run = decode_run(total * a.units);
      begin = group * run;
      end = min(begin + run, total);
      if (begin >= total) return;
      const int seq_place = begin / per_seq;    // as if all heads lay side by side: places [seq_place, ..) of one head
      const int at = __builtin_ctzll(__ballot(upto > seq_place));
      first = __builtin_amdgcn_readlane(upto - mine, at);
      b = at * each;
#pragma unroll
      for (int i = 0; i < kPlanBatch / 64; ++i) {
        const int n = __builtin_amdgcn_readlane(places[i], at);
        if (first + n > seq_place) break;       // (and b < batch: that lane holds the place)
        first += n;
        ++b;
      }
      first *= per_seq;
      if (begin == 0 && sub == 0 && tid == 0) a.first_place[a.batch] = total;
    } else {                                    // the last sequence that begins at or before the run: 64 candidates at a time
      const int total = a.first_place[a.batch];
      run = decode_run(total * a.units);
      begin = group * run;
      end = min(begin + run, total);
      if (begin >= total) return;
      for (int n = a.batch; n > 1;) {
        const int apart = (n + 63) / 64, at = lane * apart;
        const bool before = at < n && a.first_place[b + min(at, n - 1)] <= begin;
        const int skip = (__builtin_popcountll(__ballot(before)) - 1) * apart;
        b += skip;
        n = min(apart, n - skip);
      }
      first = a.first_place[b];
    }
  } else {
    if (group >= a.batch * per_seq) return;
    b = group / per_seq;
  }

  for (int pos = begin; pos < end;) {
    const int len = cached_tokens(a, b), seq = b;
    int kvh, t0 = 0, t1 = (len + kDecodeTile - 1) / kDecodeTile, place = 0;      // tiles
    bool whole = true;
    if constexpr (kSplit) {
      const int steps = decode_steps(len), seq_first = first;
      kvh = (pos - first) / (steps + kDecodeLead);
      const int head_first = first + kvh * (steps + kDecodeLead);
      const DecodePiece piece = decode_piece(head_first, steps, group, run);
      pos = head_first + steps + kDecodeLead;
      if (kvh + 1 == per_seq) {
        ++b;
        first = pos;
      }
      if (piece.t1 <= piece.t0) continue;      // the run ends before its first step
      t0 = piece.t0 * kDecodeWaves;
      t1 = min(t1, piece.t1 * kDecodeWaves);
      whole = piece.t0 == 0 && piece.t1 == steps;
      place = decode_part(piece, group) * a.units + sub;
      if (a.batch <= kPlanBatch && kvh == 0 && sub == 0 && t0 == 0 && tid == 0) a.first_place[seq] = seq_first;
    } else {
      kvh = group - b * per_seq;
      pos = end;
    }
    const int h0 = kvh * a.group + sub * kHeads;
    const int heads = min(kHeads, (kvh + 1) * a.group - h0);

    // queries: lane (g, n) holds chunk 4 c + g of head n
    uintx4 qf[kNT][kKSteps];
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int c = 0; c < kKSteps; ++c) {
        const int h = nt * 16 + r;
        qf[nt][c] = *reinterpret_cast<const uintx4*>(a.q + seq * a.q_b + (h0 + min(h, heads - 1)) * a.q_h + (4 * c + g) * 16);
      }
    floatx4 acc[kNT][kBlocks];
    float m[kNT], l[kNT];
    const int32_t* table = a.table + (int64_t)seq * a.table_stride;
    const char* k_head = a.k + kvh * a.k_h;
    const char* v_head = a.v + kvh * a.v_h;
    const int64_t page_stride = lane < 32 ? a.k_b : a.v_b, row_stride = lane < 32 ? a.k_l : a.v_l;
    int page_id, page_off;
    auto look_up = [&](int t) {               // the page of the lane's token of tile t; both halves of the wave: the same tokens
      const int tok = t * kDecodeTile + (lane & 31);
      page_id = -1;
      page_off = 0;
      if (t < t1 && tok < len) {
        const int p = (int)a.page.div(tok);
        page_off = tok - p * (int)a.page.d;
        page_id = table[p];
      }
    };
    look_up(t0 + wave);
#pragma clang loop unroll(disable)             // one copy: the first pass is not taken out of it
    for (float first = 1.f;; first = kBelow) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt) {
        m[nt] = -INFINITY;
        l[nt] = 0.f;
#pragma unroll
        for (int e = 0; e < kBlocks; ++e) acc[nt][e] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      for (int t = t0 + wave; t < t1; t += kWaves) {
        const bool valid = (unsigned)page_id < (unsigned)a.pages;
        const uint32_t live = (uint32_t)__ballot(valid);
        row_at[wave][lane >> 5][lane & 31] = valid ? page_id * page_stride + page_off * row_stride : 0;
        look_up(t + kWaves);
        uintx4 kf[2][kKSteps];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) {         // rows 8 i .. 8 i + 7 of the half, a line of 128 bytes each
            const char* row = k_head + row_at[wave][0][16 * s + 8 * i + (r & 7)] + (r >> 3) * 64 + g * 16;
#pragma unroll
            for (int c = 0; c < kKSteps; c += 2) kf[s][c + i] = load_rows<uintx4, kOnce>(row + c * 64);
          }
        uint32_t vf[2][4][kVLoads][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const char* row = v_head + row_at[wave][1][16 * s + 4 * g + j];
#pragma unroll
            for (int u = 0; u < kVLoads; ++u) {
              if constexpr (kBf16 && kD == 64) {
                const uintx2 w = load_rows<uintx2, kOnce>(row + r * 8);
                vf[s][j][u][0] = w[0]; vf[s][j][u][1] = w[1];
              } else {
                const uintx4 w = load_rows<uintx4, kOnce>(row + r * 16 + u * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e) vf[s][j][u][e] = w[e];
              }
            }
          }
        // Short rows, two waves: every load of a tile is requested before one is waited for, 1600 rows of 1 to 60 tokens 9.8 -> 9.2 us, 700 of 120 (40
        // heads on 1) 26.3 -> 25.0.  More waves fill such gaps, and the compiler's order is better: one row of 700 10.1 -> 9.6, 16 of 1000 17.9 -> 16.5.
        if constexpr (kBf16 && kWaves == 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < 2; ++s)             // lanes r < 8 want both chunks of the first rows, the others both of the second
#pragma unroll
          for (int c = 0; c < kKSteps; c += 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = kf[s][c][e], y = kf[s][c + 1][e], other = lane_xor<8>(r < 8 ? y : x);
              kf[s][c][e] = r < 8 ? x : other;
              kf[s][c + 1][e] = r < 8 ? other : y;
            }
        floatx4 sc[kNT][2];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if constexpr (kBf16) {
              sc[nt][s] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int c = 0; c < kKSteps; ++c)
                sc[nt][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[s][c]), __builtin_bit_cast(bf16x8, qf[nt][c]),
                                                                    sc[nt][s], 0, 0, 0);
            } else {                            // four sums of d / 4 products, then theirs: less than half the error of one sum of d
              floatx4 x[4] = {};
#pragma unroll
              for (int c = 0; c < kKSteps; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  x[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[s][c][e]), __uint_as_float(qf[nt][c][e]), x[e], 0, 0, 0);
              sc[nt][s] = (x[0] + x[1]) + (x[2] + x[3]);
            }
          }
        if (live != 0xffffffffu) {              // past the end, or a page that is none: no weight, whatever the rows hold
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const bool on = (live >> (16 * s + 4 * g + j)) & 1;
#pragma unroll
              for (int nt = 0; nt < kNT; ++nt) sc[nt][s][j] = on ? sc[nt][s][j] : -INFINITY;
#pragma unroll
              for (int u = 0; u < kVLoads; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) vf[s][j][u][e] = on ? vf[s][j][u][e] : 0u;
            }
        }
        bf16x8 hi[kNT], lo[kNT];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
          float top = m[nt];
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[nt][s][j]);
          top = column_max(top);
          const float old = weight_of(m[nt], top, a.scale_log2e);
          m[nt] = top;
          float sum = 0.f;
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float p = weight_of(sc[nt][s][j], top, a.scale_log2e);
              sc[nt][s][j] = p;
              sum += p;
              if constexpr (kBf16) {
                const __bf16 h = (__bf16)(p * first);
                hi[nt][4 * s + j] = h;
                lo[nt][4 * s + j] = (__bf16)(p - (float)h);
              }
            }
          l[nt] = fmaf(l[nt], old, sum);
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) acc[nt][e] *= old;
        }
        if constexpr (kBf16) {
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) {
            // eight tokens of dimension kBlocks r + e
            constexpr uint32_t kLow = 0x05040100, kHigh = 0x07060302;
            uintx4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              w[j] = __builtin_amdgcn_perm(vf[j >> 1][2 * (j & 1) + 1][0][e >> 1], vf[j >> 1][2 * (j & 1)][0][e >> 1], e & 1 ? kHigh : kLow);
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
              acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), hi[nt], acc[nt][e], 0, 0, 0);
              acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), lo[nt], acc[nt][e], 0, 0, 0);
            }
          }
        } else {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int e = 0; e < kBlocks; ++e)
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
                  acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[s][j][e >> 2][e & 3]), sc[nt][s][j], acc[nt][e], 0, 0, 0);
        }
      }
      if (!kBf16 || first == kBelow) break;
      float any = 0.f;                        // NaN if one of them is
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int e = 0; e < kBlocks; ++e)
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            any = __builtin_elementwise_maximum(__builtin_elementwise_maximum(any, acc[nt][e][i]), acc[nt][e][i + 1]);
      if (__ballot(any != any) == 0) break;
      look_up(t0 + wave);
    }

    // the waves together.  Block e, register i of lane (g, n): head n; dimension kBlocks (4 g + i) + e (bf16), 64 (e / 4) + 4 (4 g + i) +
    // e % 4 (f32)
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) {
      const int h = nt * 16 + r;
      const float sum = column_sum(l[nt]);
      if (h < heads) {
        const int row = wave * a.part_heads + h;
        if (g == 0) part_ml[row] = make_float2(m[nt], sum);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < kBlocks; e += 4) {
            const int dim = kBf16 ? kBlocks * (4 * g + i) + e : 16 * e + 4 * (4 * g + i);
            *reinterpret_cast<floatx4*>(part + row * kPitch + dim) = floatx4{acc[nt][e][i], acc[nt][e + 1][i], acc[nt][e + 2][i], acc[nt][e + 3][i]};
          }
      }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    for (int i = tid; i < heads * (kD / 4); i += kThreads) {
      const int h = i / (kD / 4), c = i % (kD / 4);
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part_ml[w * a.part_heads + h].x);
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 ml = part_ml[w * a.part_heads + h];
        const float f = weight_of(ml.x, top, a.scale_log2e);
        sum = fmaf(ml.y, f, sum);
        o += *reinterpret_cast<const floatx4*>(part + (w * a.part_heads + h) * kPitch + 4 * c) * f;
      }
      if (whole) {
        store4<kBf16>(a.out + seq * a.out_b + (h0 + h) * a.out_h + c * 4 * kElem, normalised(o, sum));
        if (a.lse && c == 0) a.lse[(int64_t)seq * a.heads_kv * a.group + h0 + h] = lse_of(top, sum, a.scale);
      } else {
        const int64_t at = (int64_t)place * a.part_heads + h;
        *reinterpret_cast<floatx4*>(a.part_o + at * kD + 4 * c) = o;
        if (c == 0) a.part_ml[at] = make_float2(top, sum);
      }
    }
    if constexpr (kSplit) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __syncthreads();
    }
  }
}

// First places of many sequences: one workgroup, a run of sequences to a thread.
__global__ __launch_bounds__(1024) void decode_plan_kernel(DecodeArgs a) {
  __shared__ int wave_sum[16];
  const int tid = threadIdx.x, each = (a.batch + 1023) / 1024, i0 = min(tid * each, a.batch), i1 = min(i0 + each, a.batch);
  int mine = 0;
  for (int i = i0; i < i1; ++i) mine += decode_places(cached_tokens(a, i));
  const int upto = (int)wave_scan((uint32_t)mine, sum_of);
  if ((tid & 63) == 63) wave_sum[tid >> 6] = upto;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = upto - mine;
  for (int w = 0; w < tid >> 6; ++w) at += wave_sum[w];
  for (int i = i0; i < i1; ++i) {
    a.first_place[i] = at * a.heads_kv;
    at += decode_places(cached_tokens(a, i));
  }
  if (tid == 1023) a.first_place[a.batch] = at * a.heads_kv;
}

// The pieces of a (sequence, query head) that more than one workgroup had a part in, added up: 4 numbers to a lane, a part to every d / 4
// lanes, four of them requested at once.  kThreads to a row: 1024 where there are few rows, whose sequences may be cut into hundreds of
// parts; 64, four rows to a workgroup, where there are many, whose sequences are cut into few if at all.
constexpr int kPartsAtOnce = 4, kCUs = 256;
template <bool kBf16, int kD, int kThreads>
__global__ __launch_bounds__(kThreads > 256 ? kThreads : 256) void decode_join_kernel(DecodeArgs a, int heads_per_unit) {
  constexpr int kAtOnce = kThreads < 256 ? 256 / kThreads : 1, kLanes = kD / 4, kRows = kThreads / kLanes, kElem = kBf16 ? 2 : 4;
  __shared__ floatx4 row_o[kAtOnce][kRows][kLanes];
  __shared__ float2 row_ml[kAtOnce][kRows];
  const int tid = threadIdx.x % kThreads, mine = threadIdx.x / kThreads;
  const int heads_q = a.heads_kv * a.group, id = min((int)blockIdx.x * kAtOnce + mine, a.batch * heads_q - 1), b = id / heads_q, head = id - b * heads_q;
  const int kvh = head / a.group, sub = (head - kvh * a.group) / heads_per_unit, h = head - kvh * a.group - sub * heads_per_unit;
  const int run = decode_run(a.first_place[a.batch] * a.units), steps = decode_steps(cached_tokens(a, b));
  const int first = a.first_place[b] + kvh * (steps + kDecodeLead);
  const int g0 = decode_first_group(first, run), g1 = decode_last_group(first, steps, run);
  const bool split = g0 != g1 && (kAtOnce == 1 || id == (int)blockIdx.x * kAtOnce + mine);
  if (kAtOnce == 1 && !split) return;
  const int c = tid % kLanes, row = tid / kLanes;
  float m = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int w0 = g0 + row; split && w0 <= g1; w0 += kRows * kPartsAtOnce) {
    float2 ml[kPartsAtOnce];
    floatx4 p[kPartsAtOnce];
#pragma unroll
    for (int j = 0; j < kPartsAtOnce; ++j) {
      const int w = min(w0 + j * kRows, g1);
      const int64_t place = (int64_t)(decode_part(decode_piece(first, steps, w, run), w) * a.units + sub) * a.part_heads + h;
      ml[j] = a.part_ml[place];
      p[j] = *reinterpret_cast<const floatx4*>(a.part_o + place * kD + 4 * c);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kPartsAtOnce; ++j) top = fmaxf(top, ml[j].x);
    const float old = weight_of(m, top, a.scale_log2e);
    m = top;
    l *= old;
    o *= old;
#pragma unroll
    for (int j = 0; j < kPartsAtOnce; ++j) {
      if (w0 + j * kRows > g1) break;
      const float f = weight_of(ml[j].x, top, a.scale_log2e);
      l = fmaf(ml[j].y, f, l);
      o += p[j] * f;
    }
  }
  row_o[mine][row][c] = o;
  if (c == 0) row_ml[mine][row] = make_float2(m, l);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  if (row > 0 || !split) return;
  float top = -INFINITY, sum = 0.f;           // (8 rows at a time: of d = 64 there are 64, more than there are registers for)
#pragma unroll 8
  for (int i = 0; i < kRows; ++i) top = fmaxf(top, row_ml[mine][i].x);
  o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = 0; i < kRows; ++i) {
    const float f = weight_of(row_ml[mine][i].x, top, a.scale_log2e);
    sum = fmaf(row_ml[mine][i].y, f, sum);
    o += row_o[mine][i][c] * f;
  }
  store4<kBf16>(a.out + b * a.out_b + head * a.out_h + c * 4 * kElem, normalised(o, sum));
  if (a.lse && c == 0) a.lse[id] = lse_of(top, sum, a.scale);
}

// Query heads that share the loads of their KV head, a unit: up to 32 (bf16), 16 (f32, whose rows take twice the registers).  Of more heads there
// are several units, whose workgroups read the rows at the same time through one L2: 64 sequences of 16384 tokens, 64 heads on 1, bf16 205 -> 148 us (each
// unit by itself -> side by side, rows kept); 16 of 8192, 160 heads on 8, f32 373 -> 291; 320 heads 545 -> 377.
// In one launch (streaming loads and neighbours in the grid -> side by side, rows kept): 500 of 700, 40 on 1, bf16 71 -> 59, 20 on 1, f32 130 -> 109; 64
// of 700, 64 on 1, bf16 16.0 -> 14.0, f32 34 -> 24; 700 of 120, 40 on 1, bf16 25.2 -> 20.9; level: one of 300, 64 on 1.
int heads_per_unit(int group, bool bf16) { return bf16 && group > 16 ? 32 : 16; }
// One workgroup of 8 waves for all of a (sequence, run of query heads): no cut, no join, one launch.  Every further 256 tokens, a tile for each wave,
// take 1 to 3 us (bf16, d = 128; one sequence of 256, 512, 768, 1024: 7.0, 7.8, 10.8, 13.0 us); so that is for calls that are short, or have a workgroup
// for every other compute unit and are not long.  One launch -> two (32 heads on 8, d = 128): one sequence of 256 tokens 7.0 -> 5.3 + 4.8 us on the device,
// of 700 9.8 -> 5.8 + 4.2 - 5.3, of 1024 13.0 -> 6.0 + 5.3; calls one after the other 7.3 -> 9.6, 9.9 -> 10.1, 13.0 -> 10.4; 64 of 200 to 1000
// 29.7 -> 28.4 + 4.1, 16 of 1000 16.2 - 17.6 -> 16.0 + 4.1.
bool is_solo(int64_t units, int row_tokens) { return row_tokens <= 768 || (row_tokens <= 1024 && units >= kCUs / 2); }
// Many short rows: workgroups of 2 waves, of which each compute unit holds more, so that the end of one overlaps others; a line between rows
// that are long beside their number and the reverse.  8 waves -> 2, 4 heads on 1, d = 128, lengths spread over their logarithm: 1600 rows of 1 to 60 tokens
// 19.2 -> 7.6 us, 1600 of 60 to 120 24.5 -> 16.2, 1024 of 20 to 500 25.0 -> 24.1, 8000 of 100 to 250 151 -> 114, 8000 of 100 to 1000 283 -> 272, 2048 of 100 to
// 1000 81 -> 85; kept at 8: 64 rows of 100 to 250 7.5 / 8.5, 1024 of 20 to 1000 (d = 64) 20 / 24.  Evenly spread: 20.5 -> 8.5, 25 -> 16.5, 30 -> 30.5, 156 ->
// 121, 364 -> 370, 99 -> 106; 7.5 / 8.6, 27.4 / 29.5.
bool has_small_workgroups(int64_t units, int row_tokens) { return units >= 2 * row_tokens; }
int64_t most_places(int batch, int heads_kv, int group, bool bf16, int row_tokens) {
  return (int64_t)batch * heads_kv * ceil_div(group, heads_per_unit(group, bf16)) * decode_places(row_tokens);
}
// Runs of a call, whatever the lengths turn out to be; as many workgroups for each as there are units.
int most_runs(int64_t places, int units) { return ceil_div(decode_groups(places), units); }
struct DecodeWs { size_t first_place, part_o, part_ml, total; };
DecodeWs carve(int batch, int groups, int part_heads, int d) {
  DecodeWs w;
  size_t o = 0;
  w.first_place = o; o += align_up((size_t)(batch + 1) * 4, 256);
  w.part_o = o; o += align_up((size_t)2 * groups * part_heads * d * 4, 256);
  w.part_ml = o; o += align_up((size_t)2 * groups * part_heads * 8, 256);
  w.total = o;
  return w;
}

template <bool kBf16, int kD, int kNT, int kWaves, bool kSplit, bool kOnce = true>
basa_status launch_kernel(const DecodeArgs& a, int groups, hipStream_t st) {
  const auto kernel = decode_kernel<kBf16, kD, kNT, kWaves, kSplit, kOnce>;
  const int lds = kWaves * a.part_heads * ((kD + 4) * 4 + 8);
  if (lds > 60 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(dynamic LDS)");
  }
  ProfScope prof(K_DECODE, st);
  kernel<<<groups, 64 * kWaves, lds, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("decode_kernel");
  return BASA_OK;
}
template <bool kBf16, int kD, int kNT>
basa_status launch(const DecodeArgs& a, int groups, hipStream_t st) {
  const int64_t units = (int64_t)a.batch * a.heads_kv * a.units;
  if (is_solo(units, a.row_tokens)) {
    const bool small = has_small_workgroups(units, a.row_tokens);
    const int rows = a.batch * a.heads_kv;
    if constexpr (!kBf16 || kNT > 1) {
      const int groups = (int)align_up(rows, 8) * a.units;
      if (a.units > 1) return small ? launch_kernel<kBf16, kD, kNT, 2, false, false>(a, groups, st)
                                    : launch_kernel<kBf16, kD, kNT, 8, false, false>(a, groups, st);
    }
    return small ? launch_kernel<kBf16, kD, kNT, 2, false>(a, rows, st) : launch_kernel<kBf16, kD, kNT, 8, false>(a, rows, st);
  }
  basa_status s = BASA_OK;
  if (a.batch > kPlanBatch) {
    ProfScope prof(K_DECODE, st);
    decode_plan_kernel<<<1, 1024, 0, st>>>(a);
    BASA_HIP_CHECK_LAUNCH("decode_plan_kernel");
  }
  if constexpr (!kBf16 || kNT > 1) s = a.units > 1 ? launch_kernel<kBf16, kD, kNT, kDecodeWaves, true, false>(a, groups, st)
                                                   : launch_kernel<kBf16, kD, kNT, kDecodeWaves, true>(a, groups, st);
  else s = launch_kernel<kBf16, kD, kNT, kDecodeWaves, true>(a, groups, st);
  if (s != BASA_OK) return s;
  ProfScope prof(K_DECODE_JOIN, st);
  const int rows = a.batch * a.heads_kv * a.group;
  if (rows <= kCUs) decode_join_kernel<kBf16, kD, 1024><<<rows, 1024, 0, st>>>(a, 16 * kNT);
  else if (rows < 4 * kCUs) decode_join_kernel<kBf16, kD, 256><<<rows, 256, 0, st>>>(a, 16 * kNT);
  else decode_join_kernel<kBf16, kD, 64><<<ceil_div(rows, 4), 256, 0, st>>>(a, 16 * kNT);
  BASA_HIP_CHECK_LAUNCH("decode_join_kernel");
  return BASA_OK;
}

}  // namespace

bool decode_takes(int batch, int heads_q, int heads_kv, bool bf16, int row_tokens) {
  return most_places(batch, heads_kv, heads_q / heads_kv, bf16, row_tokens) < INT_MAX - kDecodeMost;
}
size_t decode_workspace_bytes(int batch, int heads_q, int heads_kv, int d, bool bf16, int row_tokens) {
  const int group = heads_q / heads_kv;
  if (is_solo((int64_t)batch * heads_kv * ceil_div(group, heads_per_unit(group, bf16)), row_tokens)) return 256;
  const int hpu = heads_per_unit(group, bf16), units = ceil_div(group, hpu);
  return carve(batch, most_runs(most_places(batch, heads_kv, group, bf16, row_tokens), units) * units, std::min(group, hpu), d).total;
}

basa_status launch_decode_attn(const TensorView& q, const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width,
                               int64_t table_stride, const int32_t* lens, void* out, int64_t out_sb, int64_t out_sh, float* lse, void* ws,
                               hipStream_t st) {
  DecodeArgs a{};
  const bool bf16 = q.dtype == BASA_BF16;
  const int e = bf16 ? 2 : 4;
  a.q = static_cast<const char*>(q.ptr); a.k = static_cast<const char*>(k_pages.ptr); a.v = static_cast<const char*>(v_pages.ptr);
  a.q_b = q.stride_b * e; a.q_h = q.stride_h * e;
  a.k_b = k_pages.stride_b * e; a.k_h = k_pages.stride_h * e; a.k_l = k_pages.stride_l * e;
  a.v_b = v_pages.stride_b * e; a.v_h = v_pages.stride_h * e; a.v_l = v_pages.stride_l * e;
  a.table = table; a.table_stride = table_stride; a.lens = lens;
  a.batch = q.batch; a.heads_kv = k_pages.heads; a.group = q.heads / k_pages.heads; a.pages = k_pages.batch;
  a.row_tokens = width * k_pages.L;
  a.page = fast_div((uint32_t)k_pages.L);
  const int hpu = heads_per_unit(a.group, bf16);
  a.units = ceil_div(a.group, hpu);
  a.out = static_cast<char*>(out); a.out_b = out_sb * e; a.out_h = out_sh * e; a.lse = lse;
  const int runs = most_runs(most_places(a.batch, a.heads_kv, a.group, bf16, a.row_tokens), a.units);
  const int groups = a.units == 1 ? runs : (int)align_up(runs, 8) * a.units;
  a.part_heads = std::min(a.group, hpu);
  const DecodeWs w = carve(a.batch, runs * a.units, a.part_heads, q.d);
  char* base = static_cast<char*>(ws);
  a.first_place = reinterpret_cast<int*>(base + w.first_place);
  a.part_o = reinterpret_cast<float*>(base + w.part_o);
  a.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  a.scale = 1.0f / sqrtf((float)q.d);
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)q.d);
  if (!bf16) return q.d == 128 ? launch<false, 128, 1>(a, groups, st) : launch<false, 64, 1>(a, groups, st);
  if (hpu == 16) return q.d == 128 ? launch<true, 128, 1>(a, groups, st) : launch<true, 64, 1>(a, groups, st);
  return q.d == 128 ? launch<true, 128, 2>(a, groups, st) : launch<true, 64, 2>(a, groups, st);
}

}  // namespace basa
