// What goes on around trees of drafted tokens in a paged key-value cache: who sees whom in a tree, kept tokens moved together, sequences that go
// on from others, the pages that no one holds.
#include <algorithm>
#include <climits>
#include "common.hpp"
#include "paged_plan.hpp"

namespace basa {
namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ int sum_of(int x, int y) { return x + y; }
__device__ __forceinline__ int pages_of(const FastDiv& page, int tokens) {
  const int whole = (int)page.div(tokens);
  return whole + (whole * (int)page.d != tokens);
}

// ---- who sees whom ---------------------------------------------------------------------------------
// M(r) = {r} u M(p(r)): in two steps.  Within a run of 64 tokens, one wave: bits and the way out (the first ancestor before the run) by doubling, six
// rounds of lane exchanges.  Then a token's row is its own run's bits, those of its way out, and so on: at most one step per 64 tokens.
// Bound by latency: 2.6 us of 8 sequences of 25 tokens, as long as the shortest kernel takes; 3.9 of 200 ragged ones.
__global__ __launch_bounds__(256) void tree_masks_kernel(const int32_t* parents, const int32_t* cu, int tokens, uint64_t* masks, int words,
                                                         int64_t mask_stride, int32_t* depths) {
  extern __shared__ __attribute__((aligned(16))) uint64_t run_bits[];      // [64 words], then the ways out
  int* const way_out = reinterpret_cast<int*>(run_bits + 64 * words);
  const int tid = threadIdx.x, lane = tid & 63;
  const PackedRows rows = packed_rows(cu[blockIdx.x], cu[blockIdx.x + 1], tokens);
  const int row0 = rows.row0, n = max(rows.n, 0), fit = min(n, 64 * words);
  for (int run = tid >> 6; run * 64 < fit; run += 4) {
    const int r = run * 64 + lane;
    int p = r < fit ? parents[row0 + r] : -1;
    if (p >= r) p = -1;
    uint64_t bits = 1ull << lane;
    int up = p >= run * 64 ? p - run * 64 : -1, out = p < run * 64 ? max(p, -1) : -1;
#pragma unroll
    for (int k = 0; k < 6; ++k) {
      const int from = max(up, 0), up2 = __shfl(up, from), out2 = __shfl(out, from);
      const uint64_t bits2 = __shfl(bits, from);
      if (up >= 0) {
        bits |= bits2;
        out = out2;
        up = up2;
      }
    }
    run_bits[r] = bits;
    way_out[r] = out;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  for (int r = tid; r < n; r += 256) {
    int at = r < fit ? r : -1, depth = -1;
    uint64_t* const row = masks + (row0 + r) * mask_stride;
    for (int w = words - 1; w >= 0; --w) {
      uint64_t bits = 0;
      if (at >= 0 && at >> 6 == w) {
        bits = run_bits[at];
        depth += __popcll(bits);
        at = way_out[at];
      }
      row[w] = bits;
    }
    if (depths) depths[row0 + r] = depth;
  }
}

// ---- kept tokens moved together --------------------------------------------------------------------
// Token start + keep[j] of a sequence to start + j, in place.  keep ascends, so keep[j] >= j: no move writes what a later one reads, and what one reads is written by
// a later one or itself.  So whoever moves the same bytes of every row needs no one else, if of any two rows it reads the first before it writes the second: a lane in the
// order of the list, or a workgroup that reads many rows before it writes them.
struct CompactArgs {
  char *k, *v;
  int64_t k_b, k_h, k_l, v_b, v_h, v_l;     // bytes
  const int32_t *table, *start, *keep, *count, *lens;       // lens: tokens that a sequence holds, or null: as many as its row has room for
  int64_t table_stride, keep_stride;
  int width, most, pages, row_bits, parts;  // bytes of a row of one head; parts of K and V of a token: of a lane or a workgroup
  FastDiv page;
};
// Tokens of a sequence that may be read.  (Entries of its row behind them may be the ids of pages that others have by now.)
__device__ __forceinline__ int tokens_held(const CompactArgs& a, int seq) {
  const int room = a.width * (int)a.page.d;      // at most 2^30
  return a.lens ? min(a.lens[seq], room) : room;
}
// Where move j of a sequence reads and writes in K or V, from the head's row on; -1: no move.
struct Move { int64_t from, to; };
__device__ __forceinline__ Move move_of(const CompactArgs& a, int seq, int held, int start, int j, int64_t page_bytes, int64_t row_bytes) {
  const int kept = a.keep[(int64_t)seq * a.keep_stride + j];
  const int32_t* const row = a.table + (int64_t)seq * a.table_stride;
  const int64_t from = (int64_t)start + kept, to = (int64_t)start + j;
  if (start < 0 || kept <= j || from >= held) return {-1, -1};
  const int from_page = (int)a.page.div((uint32_t)from), to_page = (int)a.page.div((uint32_t)to);
  const int from_id = row[from_page], to_id = row[to_page];
  if ((unsigned)from_id >= (unsigned)a.pages || (unsigned)to_id >= (unsigned)a.pages) return {-1, -1};
  return {from_id * page_bytes + (from - (int64_t)from_page * a.page.d) * row_bytes, to_id * page_bytes + (to - (int64_t)to_page * a.page.d) * row_bytes};
}

// Short lists, the paths of trees: a lane to every 16 bytes of a token.  Bound by latency: 3.5 us of 64 sequences with paths of some 5 of 16 tokens.
constexpr int kMoves = 256, kAtOnce = 8;
__global__ __launch_bounds__(256) void compact_kernel(CompactArgs a) {
  __shared__ Move moves[2][kMoves];         // K, V
  const int seq = blockIdx.x, tid = threadIdx.x, part = blockIdx.y * 256 + tid;
  const int count = min(max(a.count[seq], 0), a.most), start = a.start[seq], held = tokens_held(a, seq);
  const bool is_v = part >= a.parts;
  const int c = is_v ? part - a.parts : part;
  const int64_t h = c >> (a.row_bits - 4), in_row = (c & ((1 << (a.row_bits - 4)) - 1)) * 16;
  char* const rows = (is_v ? a.v + h * a.v_h : a.k + h * a.k_h) + in_row;
  const bool works = part < 2 * a.parts;
  for (int j0 = 0; j0 < count; j0 += kMoves) {
    const int n = min(count - j0, kMoves);
    if (tid < n) {
      moves[0][tid] = move_of(a, seq, held, start, j0 + tid, a.k_b, a.k_l);
      moves[1][tid] = move_of(a, seq, held, start, j0 + tid, a.v_b, a.v_l);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
    for (int i0 = 0; works && i0 < n; i0 += kAtOnce) {
      uintx4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) x[i] = *reinterpret_cast<const uintx4*>(rows + max(moves[is_v][min(i0 + i, n - 1)].from, (int64_t)0));
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (i0 + i < n && moves[is_v][i0 + i].to >= 0) *reinterpret_cast<uintx4*>(rows + moves[is_v][i0 + i].to) = x[i];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
  }
}

// Long lists: a workgroup to every 128 bytes of a token's K or V, eight lanes to a row, eight rows to each of them read before one is written, a move to every thread.  The
// next rows are read while these are written; what their places come from was asked for a turn and two turns earlier.  Bound by the memory, or by the longest list, whose
// workgroups take turn after turn: 12 sequences of 2000 to 16000 tokens, two thirds kept, 446 MB in 120 us, 3.7 TB/s (a lane to 16 bytes, as for short lists: 2400 us).
constexpr int kLine = 128, kLinesAtOnce = 8;
template <int kThreads>
__global__ __launch_bounds__(kThreads, 4) void compact_lines_kernel(CompactArgs a) {
  __shared__ Move moves[3][kThreads];         // of the rows that are written, of those that are read, of the next
  const int seq = blockIdx.x / (2 * a.parts), part = blockIdx.x - seq * 2 * a.parts, tid = threadIdx.x;
  const int count = min(max(a.count[seq], 0), a.most), start = a.start[seq], held = tokens_held(a, seq);
  if (count == 0) return;
  const bool is_v = part >= a.parts;
  const int c = is_v ? part - a.parts : part;
  const int64_t h = c >> (a.row_bits - 7), in_row = (c & ((1 << (a.row_bits - 7)) - 1)) * kLine + (tid & 7) * 16;
  char* const rows = (is_v ? a.v + h * a.v_h : a.k + h * a.k_h) + in_row;
  const int64_t page_bytes = is_v ? a.v_b : a.k_b, row_bytes = is_v ? a.v_l : a.k_l;
  const int32_t* const keep = a.keep + (int64_t)seq * a.keep_stride;
  const int32_t* const table = a.table + (int64_t)seq * a.table_stride;
  // A thread's move of the turn that begins with j0, in three steps: the kept token, the ids of its pages, its place.  (No branches, so that nothing waits within one.)
  struct Kept { int j, token; };
  struct Pages { int64_t from, to; int from_page, to_page, from_id, to_id; bool valid; };
  auto ask_token = [&](int j0) {
    const int j = j0 + tid;
    return Kept{j, keep[min(j, count - 1)]};
  };
  auto ask_pages = [&](Kept k) {
    Pages p;
    p.from = (int64_t)start + k.token;
    p.to = (int64_t)start + k.j;
    p.valid = k.j < count && start >= 0 && k.token > k.j && p.from < held;
    p.from_page = (int)a.page.div(p.valid ? (uint32_t)p.from : 0u);
    p.to_page = (int)a.page.div(p.valid ? (uint32_t)p.to : 0u);
    p.from_id = table[p.from_page];
    p.to_id = table[p.to_page];
    return p;
  };
  auto put_move = [&](Pages p, int side) {
    const bool valid = p.valid && (unsigned)p.from_id < (unsigned)a.pages && (unsigned)p.to_id < (unsigned)a.pages;
    moves[side][tid] = valid ? Move{p.from_id * page_bytes + (p.from - (int64_t)p.from_page * a.page.d) * row_bytes,
                                    p.to_id * page_bytes + (p.to - (int64_t)p.to_page * a.page.d) * row_bytes} : Move{-1, -1};
  };
  auto read = [&](uintx4 (&x)[kLinesAtOnce], int side) {
#pragma unroll
    for (int i = 0; i < kLinesAtOnce; ++i) x[i] = *reinterpret_cast<const uintx4*>(rows + max(moves[side][i * (kThreads / 8) + (tid >> 3)].from, (int64_t)0));
  };
  auto write = [&](const uintx4 (&x)[kLinesAtOnce], int side) {
#pragma unroll
    for (int i = 0; i < kLinesAtOnce; ++i) {
      const int64_t to = moves[side][i * (kThreads / 8) + (tid >> 3)].to;
      if (to >= 0) *reinterpret_cast<uintx4*>(rows + to) = x[i];
    }
  };
  // vmcnt(0) lgkmcnt(0): my rows are here, and my move is in the LDS; after the barrier everyone's
  auto meet = [&] {
    __builtin_amdgcn_s_waitcnt(0x0070);
    asm volatile("" ::: "memory");
    __syncthreads();
  };
  uintx4 x[kLinesAtOnce], y[kLinesAtOnce];
  int side = 0;
  auto next = [&](int at) { return at == 2 ? 0 : at + 1; };
  Kept kept = ask_token(0);
  Pages pages = ask_pages(kept);
  kept = ask_token(kThreads);
  put_move(pages, 0);
  pages = ask_pages(kept);
  kept = ask_token(2 * kThreads);
  meet();
  read(x, 0);
  // The rows before j0 are in `mine` or on their way there; those from j0 on go to `others`.  False: there are none.
  auto turn = [&](uintx4 (&mine)[kLinesAtOnce], uintx4 (&others)[kLinesAtOnce], int j0) {
    const int ahead = next(side);
    put_move(pages, ahead);
    meet();
    pages = ask_pages(kept);                    // of j0 + kThreads
    kept = ask_token(j0 + 2 * kThreads);
    if (j0 < count) read(others, ahead);
    write(mine, side);
    side = ahead;
    return j0 < count;
  };
  for (int j0 = kThreads; turn(x, y, j0) && turn(y, x, j0 + kThreads); j0 += 2 * kThreads) {
  }
}
// Which lists are short: a workgroup to a line costs 5 ns whatever it moves, a lane that goes down a list waits 0.1 us for eight moves while there is no other to run.  Short / long, of 8
// sequences (8 heads, d = 128, bf16) lists of 64 10.6 / 8.1 us; of 64 sequences 43 8.9 / 13.3, 85 15.6 / 14.9, 171 30 / 20; of 200 85 24 / 43, 171 55.3 / 55.4, 343 124 / 98.
bool is_short(int most, int64_t lines) { return most <= 48 + lines / 48; }

// ---- sequences that go on from others --------------------------------------------------------------
// New sequence j shares the whole pages of its parent.  The page that is not full, if there is one, goes to the first new sequence of the parent; each
// further one gets the next of the free pages, and a copy of its tokens to make.  Every workgroup finds the first ones (a minimum, whatever the order of
// its parts) and the running sum of the pages for itself, then writes its rows.  Bound by latency: 3.7 us of 64 from 8, 5.8 of 512 from 512.
struct ForkArgs {
  const int32_t *table, *lens, *parents, *free_pages;
  int64_t table_stride, new_stride;
  int32_t *new_table, *new_lens, *copies, *pages;
  int width, n_old, n_new, n_free;
  FastDiv page;
};
constexpr int kMaxForkSeqs = 8192;
constexpr int kShares = -1, kNotServed = -2;
__global__ __launch_bounds__(256) void page_fork_kernel(ForkArgs a) {
  extern __shared__ int fork_words[];
  __shared__ int wave_sum[4];
  int* const first = fork_words;              // of an old sequence: its first new one
  int* const place = fork_words + a.n_old;    // of a new sequence: its place among the free pages, or one of the above
  const int tid = threadIdx.x, each = (a.n_new + 255) / 256, j0 = min(tid * each, a.n_new), j1 = min(j0 + each, a.n_new);
  for (int i = tid; i < a.n_old; i += 256) first[i] = INT_MAX;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  for (int j = tid; j < a.n_new; j += 256) {
    const int p = a.parents[j];
    if ((unsigned)p < (unsigned)a.n_old) atomicMin(&first[p], j);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int room = a.width * (int)a.page.d;
  auto tokens_of = [&](int p) { return (unsigned)p < (unsigned)a.n_old ? min(max(a.lens[p], 0), room) : 0; };
  for (int j = tid; j < a.n_new; j += 256) {
    const int p = a.parents[j], len = tokens_of(p);
    place[j] = len != (int)(a.page.div(len) * a.page.d) && first[p] != j;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int mine = 0;
  for (int j = j0; j < j1; ++j) mine += place[j];
  const int upto = (int)wave_scan((uint32_t)mine, sum_of);
  if ((tid & 63) == 63) wave_sum[tid >> 6] = upto;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = upto - mine, asked = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < tid >> 6) at += wave_sum[w];
    asked += wave_sum[w];
  }
  for (int j = j0; j < j1; ++j) {
    const int need = place[j];
    place[j] = need ? (at < a.n_free ? at : kNotServed) : kShares;
    at += need;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    a.pages[0] = min(asked, a.n_free);
    a.pages[1] = asked;
  }
  // a row to a wave at a time
  const int lane = tid & 63;
  for (int j = blockIdx.x * 4 + (tid >> 6); j < a.n_new; j += gridDim.x * 4) {
    const int p = a.parents[j], got = place[j], len = got == kNotServed ? 0 : tokens_of(p);
    const int held = pages_of(a.page, len), whole = (int)a.page.div(len), fresh = got >= 0 ? a.free_pages[got] : -1;
    const int32_t* const from = a.table + (int64_t)p * a.table_stride;
    int32_t* const to = a.new_table + (int64_t)j * a.new_stride;
    for (int i = lane; i < held; i += 64) to[i] = got >= 0 && i == whole ? fresh : from[i];
    if (lane == 0) {
      a.new_lens[j] = len;
      a.copies[3 * j] = got >= 0 ? from[whole] : -1;
      a.copies[3 * j + 1] = fresh;
      a.copies[3 * j + 2] = got >= 0 ? len - whole * (int)a.page.d : 0;
    }
  }
}

// The first tokens of a page to the same places of another: a 16-byte chunk of K and of V to a lane, in the order of memory.  56 copies of up to 64 tokens 4.5 us.
struct CopyArgs {
  char *k, *v;
  int64_t k_b, k_h, k_l, v_b, v_h, v_l;     // bytes
  const int32_t* copies;
  int pages, page, heads, chunk_bits, by_token;        // by_token: heads of a token side by side
  FastDiv inner;                            // tokens of a page, or heads
};
__global__ __launch_bounds__(256) void cache_copy_kernel(CopyArgs a) {
  const int32_t* const c = a.copies + 3 * (int64_t)blockIdx.x;
  const int from = c[0], to = c[1], tokens = min(max(c[2], 0), a.page);
  if ((unsigned)from >= (unsigned)a.pages || (unsigned)to >= (unsigned)a.pages || from == to) return;
  // (Less than 2^31 of them; a lane's number passes that on its way out.)
  const uint32_t items = (uint32_t)((a.by_token ? tokens : a.page) * a.heads) << a.chunk_bits;
  for (uint32_t i = blockIdx.y * 256 + threadIdx.x; i < items; i += gridDim.y * 256) {
    const int row = (int)(i >> a.chunk_bits), outer = (int)a.inner.div(row), in = row - outer * (int)a.inner.d;
    const int64_t h = a.by_token ? in : outer, t = a.by_token ? outer : in, at = (i & ((1 << a.chunk_bits) - 1)) * 16;
    if (t >= tokens) continue;
    const uintx4 k = *reinterpret_cast<const uintx4*>(a.k + from * a.k_b + h * a.k_h + t * a.k_l + at);
    const uintx4 v = *reinterpret_cast<const uintx4*>(a.v + from * a.v_b + h * a.v_h + t * a.v_l + at);
    *reinterpret_cast<uintx4*>(a.k + to * a.k_b + h * a.k_h + t * a.k_l + at) = k;
    *reinterpret_cast<uintx4*>(a.v + to * a.v_b + h * a.v_h + t * a.v_l + at) = v;
  }
}

// ---- the pages that no one holds -------------------------------------------------------------------
// A bit for every page, set by the table rows as far as their lengths need pages; then the ids whose bit is not set, in order.  Bound by latency: 6.7 us in one workgroup of
// 64 sequences of up to 500 pages, three launches of 2.2, 5.0 and 7.7 us of 2000 of up to 1250.
struct FreeArgs {
  const int32_t *table, *lens;
  int64_t table_stride;
  int n, row_tokens, pages, words;          // words of 32 bits
  int32_t *free_pages, *count;
  uint8_t* used;                            // workspace: a byte for every page, up to a multiple of 32
  int lanes;                                // of one workgroup: lanes of a wave for a row, a power of two; 0: a row is wider than a wave
  FastDiv page;
};
// Marks the pages of kRows rows, `apart` entries one behind the other, by a wave: 8 / kRows entries of each to a lane asked for at once.
template <int kRows, class Mark>
__device__ __forceinline__ void mark_rows(const FreeArgs& a, const int32_t* row, int64_t apart, const int (&held)[kRows], Mark mark) {
  constexpr int kEntries = 8 / kRows;
  int most = held[0];
#pragma unroll
  for (int r = 1; r < kRows; ++r) most = max(most, held[r]);
  for (int first = 0; first < most; first += 64 * kEntries) {                    // (as many turns for every lane)
    const int p0 = first + (threadIdx.x & 63);
    int id[kRows][kEntries];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < kEntries; ++i) id[r][i] = p0 + 64 * i < held[r] ? row[r * apart + p0 + 64 * i] : -1;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < kEntries; ++i)
        if ((unsigned)id[r][i] < (unsigned)a.pages) mark(id[r][i]);
  }
}
__device__ __forceinline__ int held_pages(const FreeArgs& a, int len) { return pages_of(a.page, min(max(len, 0), a.row_tokens)); }
// The free pages of words [first, first + n), which are in the LDS (the last word's bits past the end are set), by the whole workgroup, from place `at` of the list on.  Returns
// the place behind them.
template <int kThreads>
__device__ __forceinline__ int list_free(const FreeArgs& a, const uint32_t* used, int first, int n, int at, int* wave_sum) {
  constexpr int kGroupWaves = kThreads / 64;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int each = (n + kGroupWaves - 1) / kGroupWaves, w0 = min(wave * each, n), w1 = min(w0 + each, n);       // words of a wave
  int mine = 0;
  for (int w = w0 + lane; w < w1; w += 64) mine += __popc(~used[w]);
  const int sum = __builtin_amdgcn_readlane((int)wave_scan((uint32_t)mine, sum_of), 63);
  if (lane == 0) wave_sum[wave] = sum;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int all = at;
#pragma unroll
  for (int w = 0; w < kGroupWaves; ++w) {
    if (w < wave) at += wave_sum[w];
    all += wave_sum[w];
  }
  for (int w = w0; w < w1; w += 2) {           // 64 pages at a time
    const bool free = w + (lane >> 5) < w1 && !(used[min(w + (lane >> 5), w1 - 1)] >> (lane & 31) & 1);
    const uint64_t which = __ballot(free);
    if (free) a.free_pages[at + __popcll(which & ((1ull << lane) - 1))] = (first + w) * 32 + lane;
    at += __popcll(which);
  }
  return all;
}
__device__ __forceinline__ uint32_t past_the_end(const FreeArgs& a, int word) {
  const int left = a.pages - word * 32;
  return left >= 32 ? 0u : ~0u << left;
}
__global__ __launch_bounds__(1024) void page_free_kernel(FreeArgs a) {
  extern __shared__ uint32_t used[];
  __shared__ int wave_sum[16];
  const int wave = threadIdx.x >> 6;
  for (int w = threadIdx.x; w < a.words; w += 1024) used[w] = past_the_end(a, w);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  auto mark = [&](int id) { atomicOr(&used[id >> 5], 1u << (id & 31)); };
  if (a.lanes > 0) {                            // narrow rows: several to a wave, eight loads at once
    constexpr int kLoads = 8;
    const int per_wave = 64 / a.lanes, lane = threadIdx.x & 63, p = lane & (a.lanes - 1);
    for (int i0 = 0; i0 < a.n; i0 += 16 * kLoads * per_wave) {
      int held[kLoads], id[kLoads];              // (no load stands in a branch: they would be waited for one after the other)
      const int i = i0 + wave * kLoads * per_wave + lane / a.lanes;
#pragma unroll
      for (int r = 0; r < kLoads; ++r) held[r] = a.lens[min(i + r * per_wave, a.n - 1)];
#pragma unroll
      for (int r = 0; r < kLoads; ++r) {
        held[r] = i + r * per_wave < a.n ? held_pages(a, held[r]) : 0;
        id[r] = a.table[(int64_t)min(i + r * per_wave, a.n - 1) * a.table_stride + min(p, max(held[r] - 1, 0))];
      }
#pragma unroll
      for (int r = 0; r < kLoads; ++r) id[r] = p < held[r] ? id[r] : -1;
#pragma unroll
      for (int r = 0; r < kLoads; ++r)
        if ((uint32_t)id[r] < (uint32_t)a.pages) mark(id[r]);
    }
  } else for (int i0 = wave; i0 < a.n; i0 += 1024) {          // every 16th row to a wave: 64 lengths at once, four rows at a time
    const int i = i0 + 16 * (threadIdx.x & 63), mine = i < a.n ? held_pages(a, a.lens[i]) : 0;
    for (int r = 0; r < 64 && i0 + 16 * r < a.n; r += 4) {
      const int held[4] = {__builtin_amdgcn_readlane(mine, r), __builtin_amdgcn_readlane(mine, r + 1), __builtin_amdgcn_readlane(mine, r + 2),
                           __builtin_amdgcn_readlane(mine, r + 3)};
      mark_rows(a, a.table + (int64_t)(i0 + 16 * r) * a.table_stride, 16 * a.table_stride, held, mark);
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int all = list_free<1024>(a, used, 0, a.words, 0, wave_sum);
  if (threadIdx.x == 0) *a.count = all;
}
// Over the device a byte for every page: stores of ones need no order, and atomics on bits, which go past the XCDs' caches, took 18 of 26 us of a call of 2000 rows.
__global__ __launch_bounds__(256) void free_clear_kernel(FreeArgs a) {
  const int p0 = (blockIdx.x * 256 + threadIdx.x) * 16;
  if (p0 >= a.words * 32) return;
  uintx4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = a.pages - p0 - 4 * i;      // (the bytes past the last page are ones)
    x[i] = left >= 4 ? 0u : left <= 0 ? 0x01010101u : 0x01010101u << (8 * left);
  }
  *reinterpret_cast<uintx4*>(a.used + p0) = x;
}
__global__ __launch_bounds__(256) void free_mark_kernel(FreeArgs a) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= a.n) return;
  const int held[1] = {held_pages(a, a.lens[i])};
  mark_rows(a, a.table + (int64_t)i * a.table_stride, 0, held, [&](int id) { a.used[id] = 1; });
}
// A workgroup counts the free pages before its words for itself.
constexpr int kListWords = 2048;
__global__ __launch_bounds__(1024) void free_list_kernel(FreeArgs a, int words_each) {
  __shared__ int before[16], wave_sum[16];
  __shared__ uint32_t used[kListWords];
  const int first = blockIdx.x * words_each, n = min(words_each, a.words - first), tid = threadIdx.x;
  int mine = 0;
  const uintx4* const bytes = reinterpret_cast<const uintx4*>(a.used);
  constexpr int kLoads = 8;
  for (int c0 = 0; c0 < 2 * first; c0 += 1024 * kLoads) {     // 16 pages each
    uintx4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = bytes[min(c0 + 1024 * i + tid, 2 * a.words - 1)];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) mine += c0 + 1024 * i + tid < 2 * first ? 16 - __popc(x[i][0]) - __popc(x[i][1]) - __popc(x[i][2]) - __popc(x[i][3]) : 0;
  }
  for (int w = (tid >> 6) * 2; w < n; w += 32) {              // 64 pages at a time as bits
    const uint64_t bits = __ballot(w + (tid >> 5 & 1) < n && a.used[(int64_t)(first + min(w + (tid >> 5 & 1), n - 1)) * 32 + (tid & 31)]);
    if ((tid & 31) == 0 && w + (tid >> 5 & 1) < n) used[w + (tid >> 5 & 1)] = (uint32_t)(tid & 32 ? bits >> 32 : bits);
  }
  const int sum = __builtin_amdgcn_readlane((int)wave_scan((uint32_t)mine, sum_of), 63);
  if ((tid & 63) == 0) before[tid >> 6] = sum;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) at += before[w];
  const int all = list_free<1024>(a, used, first, n, at, wave_sum);
  if (first + n == a.words && tid == 0) *a.count = all;
}
// In one workgroup, or in three launches over the device.
int lanes_of_row(int width) {                   // 0: more than a wave
  int lanes = width <= 64 ? 1 : 0;
  while (lanes && lanes < width) lanes *= 2;
  return lanes;
}
// By the wave's marks that there may be, 64 entries each: 1000 rows of up to 63 pages 17.4 us in one workgroup, 11 over the device; 250 of up to 250, whose marks come in whole waves, 8.9.
bool free_in_one(int n_seq, int width, int n_pages) {
  const int lanes = lanes_of_row(width);
  const int64_t entries = (int64_t)n_seq * (lanes ? lanes : align_up(width, 64));
  return n_pages <= (1 << 18) && entries <= (n_seq <= 256 ? 1 << 16 : 1 << 15);
}

}  // namespace

basa_status launch_tree_masks(const int32_t* parents, const int32_t* cu, int n, int tokens, int64_t* masks, int words, int64_t mask_stride,
                              int32_t* depths, hipStream_t st) {
  if (n == 0) return BASA_OK;
  ProfScope prof(K_PAGED, st);
  tree_masks_kernel<<<n, 256, words * 64 * 12, st>>>(parents, cu, tokens, reinterpret_cast<uint64_t*>(masks), words, mask_stride, depths);
  BASA_HIP_CHECK_LAUNCH("tree_masks_kernel");
  return BASA_OK;
}

// A launch has less than 2^32 threads.
bool compact_takes(int n, const TensorView& k) {
  return n <= 1 << 22 && (int64_t)n * k.heads * (k.d * (k.dtype == BASA_BF16 ? 2 : 4) / kLine) * 2 < (1 << 23);
}
basa_status launch_cache_compact(const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width, int64_t table_stride,
                                 const int32_t* lens, const int32_t* start, const int32_t* keep, int most, int64_t keep_stride, const int32_t* count,
                                 int n, hipStream_t st) {
  if (n == 0 || most == 0) return BASA_OK;
  CompactArgs a{};
  const int e = k_pages.dtype == BASA_BF16 ? 2 : 4;
  a.k = static_cast<char*>(const_cast<void*>(k_pages.ptr)); a.v = static_cast<char*>(const_cast<void*>(v_pages.ptr));
  a.k_b = k_pages.stride_b * e; a.k_h = k_pages.stride_h * e; a.k_l = k_pages.stride_l * e;
  a.v_b = v_pages.stride_b * e; a.v_h = v_pages.stride_h * e; a.v_l = v_pages.stride_l * e;
  a.table = table; a.lens = lens; a.start = start; a.keep = keep; a.count = count; a.table_stride = table_stride; a.keep_stride = keep_stride;
  a.width = width; a.pages = k_pages.batch;
  most = std::min(most, width * k_pages.L);       // entry j moves to j or further on: beyond the row none does (and j stays below 2^30)
  a.most = most;
  while ((1 << a.row_bits) < k_pages.d * e) ++a.row_bits;
  a.page = fast_div((uint32_t)k_pages.L);
  ProfScope prof(K_PAGED, st);
  const int64_t lines = ((int64_t)n * k_pages.heads * 2) << (a.row_bits - 7);
  if (is_short(most, lines)) {
    a.parts = k_pages.heads << (a.row_bits - 4);
    compact_kernel<<<dim3(n, ceil_div(2 * a.parts, 256)), 256, 0, st>>>(a);
    BASA_HIP_CHECK_LAUNCH("compact_kernel");
  } else {
    a.parts = k_pages.heads << (a.row_bits - 7);
    // few long lists: large turns, fewer of them (one of 40000 tokens 118 -> 112 us, 15 of 1000 to 8000 51.6 -> 49.4; but 64 of 1500 90 -> 94)
    if (lines >= 512) compact_lines_kernel<512><<<(int)lines, 512, 0, st>>>(a);
    else compact_lines_kernel<1024><<<(int)lines, 1024, 0, st>>>(a);
    BASA_HIP_CHECK_LAUNCH("compact_lines_kernel");
  }
  return BASA_OK;
}

bool page_fork_takes(int n_old, int n_new) { return n_old <= kMaxForkSeqs && n_new <= kMaxForkSeqs; }
basa_status launch_page_fork(const int32_t* table, int width, int64_t table_stride, const int32_t* lens, int n_old, int page,
                             const int32_t* parents, int n_new, const int32_t* free_pages, int n_free, int32_t* new_table, int64_t new_stride,
                             int32_t* new_lens, int32_t* copies, int32_t* pages, hipStream_t st) {
  ForkArgs a{};
  a.table = table; a.lens = lens; a.parents = parents; a.free_pages = free_pages; a.table_stride = table_stride; a.new_stride = new_stride;
  a.new_table = new_table; a.new_lens = new_lens; a.copies = copies; a.pages = pages; a.width = width; a.n_old = n_old; a.n_new = n_new;
  a.n_free = n_free; a.page = fast_div((uint32_t)page);
  const int lds = std::max((n_old + n_new) * 4, 16);
  if (lds > 60 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&page_fork_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(dynamic LDS)");
  }
  ProfScope prof(K_PAGED, st);
  page_fork_kernel<<<std::min(std::max(ceil_div(n_new, 4), 1), 512), 256, lds, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("page_fork_kernel");
  return BASA_OK;
}

basa_status launch_cache_copy(const TensorView& k_pages, const TensorView& v_pages, const int32_t* copies, int n, hipStream_t st) {
  if (n == 0) return BASA_OK;
  CopyArgs a{};
  const int e = k_pages.dtype == BASA_BF16 ? 2 : 4;
  a.k = static_cast<char*>(const_cast<void*>(k_pages.ptr)); a.v = static_cast<char*>(const_cast<void*>(v_pages.ptr));
  a.k_b = k_pages.stride_b * e; a.k_h = k_pages.stride_h * e; a.k_l = k_pages.stride_l * e;
  a.v_b = v_pages.stride_b * e; a.v_h = v_pages.stride_h * e; a.v_l = v_pages.stride_l * e;
  a.copies = copies; a.pages = k_pages.batch; a.page = k_pages.L; a.heads = k_pages.heads;
  while ((16 << a.chunk_bits) < k_pages.d * e) ++a.chunk_bits;
  a.by_token = k_pages.stride_h < k_pages.stride_l;
  a.inner = fast_div((uint32_t)(a.by_token ? a.heads : a.page));
  const int64_t items = (int64_t)a.page * a.heads << a.chunk_bits;
  ProfScope prof(K_PAGED, st);
  cache_copy_kernel<<<dim3(n, (int)std::min<int64_t>((items + 511) / 512, 64)), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("cache_copy_kernel");
  return BASA_OK;
}

size_t page_free_workspace_bytes(int n_seq, int width, int n_pages) {
  return free_in_one(n_seq, width, n_pages) ? 256 : align_up((size_t)ceil_div(n_pages, 32) * 32, 256);
}
basa_status launch_page_free(const int32_t* table, int width, int64_t table_stride, const int32_t* lens, int n_seq, int page, int n_pages,
                             int32_t* free_pages, int32_t* count, void* ws, hipStream_t st) {
  FreeArgs a{};
  a.table = table; a.lens = lens; a.table_stride = table_stride; a.n = n_seq; a.row_tokens = width * page; a.pages = n_pages;
  a.words = ceil_div(n_pages, 32); a.free_pages = free_pages; a.count = count; a.used = static_cast<uint8_t*>(ws);
  a.page = fast_div((uint32_t)page);
  a.lanes = lanes_of_row(width);
  ProfScope prof(K_PAGED, st);
  if (free_in_one(n_seq, width, n_pages)) {
    page_free_kernel<<<1, 1024, std::max(a.words * 4, 16), st>>>(a);
    BASA_HIP_CHECK_LAUNCH("page_free_kernel");
    return BASA_OK;
  }
  free_clear_kernel<<<ceil_div(2 * a.words, 256), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("free_clear_kernel");
  if (n_seq > 0) {
    free_mark_kernel<<<ceil_div(n_seq, 4), 256, 0, st>>>(a);
    BASA_HIP_CHECK_LAUNCH("free_mark_kernel");
  }
  const int groups = std::max(std::min(ceil_div(a.words, 64), 128), ceil_div(a.words, kListWords)), each = ceil_div(a.words, groups);
  free_list_kernel<<<ceil_div(a.words, each), 1024, 0, st>>>(a, each);
  BASA_HIP_CHECK_LAUNCH("free_list_kernel");
  return BASA_OK;
}

}  // namespace basa
