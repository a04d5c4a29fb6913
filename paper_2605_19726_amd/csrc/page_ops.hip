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
// Bound by latency.
__global__ __launch_bounds__(256) void tree_masks_kernel(const int32_t* parents, const int32_t* cu, int tokens, uint64_t* masks, int words,
                                                         int64_t mask_stride, int32_t* depths) {
  extern __shared__ __attribute__((aligned(16))) uint64_t run_bits[];      // [64 words], then the ways out
  int* const way_out = reinterpret_cast<int*>(run_bits + 64 * words);
  const int tid = threadIdx.x, lane = tid & 63;
  const int row0 = min(max(cu[blockIdx.x], 0), tokens), n = max(min(cu[blockIdx.x + 1], tokens) - row0, 0), fit = min(n, 64 * words);
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
// Token start + keep[j] of a sequence to start + j, in place.  keep ascends, so keep[j] >= j: no move writes what a later one reads, and each
// has to read before the one that writes there, which is a later one or itself.  So a lane that has the same 16 bytes of every row, and moves them in
// order, needs no one else.
struct CompactArgs {
  char *k, *v;
  int64_t k_b, k_h, k_l, v_b, v_h, v_l;     // bytes
  const int32_t *table, *start, *keep, *count;
  int64_t table_stride, keep_stride;
  int width, most, pages, chunk_bits, chunks;          // 16-byte chunks of one token: heads << chunk_bits
  FastDiv page;
};
constexpr int kMoves = 256, kAtOnce = 8;
__global__ __launch_bounds__(256) void compact_kernel(CompactArgs a) {
  __shared__ int64_t from_at[2][kMoves], to_at[2][kMoves];          // K, V; negative: no move
  const int seq = blockIdx.x, tid = threadIdx.x, chunk = blockIdx.y * 256 + tid;
  const int count = min(max(a.count[seq], 0), a.most), start = a.start[seq];
  const bool is_v = chunk >= a.chunks;
  const int c = is_v ? chunk - a.chunks : chunk;
  const int64_t h = c >> a.chunk_bits, in_row = (c & ((1 << a.chunk_bits) - 1)) * 16;
  char* const rows = (is_v ? a.v + h * a.v_h : a.k + h * a.k_h) + in_row;
  const bool works = chunk < 2 * a.chunks;
  const int64_t room = (int64_t)a.width * a.page.d;
  auto page_of = [&](int64_t tok, int* off) {
    if (tok < 0 || tok >= room) return -1;
    const int p = (int)a.page.div((uint32_t)tok);
    *off = (int)tok - p * (int)a.page.d;
    return a.table[(int64_t)seq * a.table_stride + p];
  };
  for (int j0 = 0; j0 < count; j0 += kMoves) {
    const int n = min(count - j0, kMoves);
    if (tid < n) {
      const int j = j0 + tid, kept = a.keep[(int64_t)seq * a.keep_stride + j];
      int from_off = 0, to_off = 0;
      const int from = page_of((int64_t)start + kept, &from_off), to = page_of((int64_t)start + j, &to_off);
      const bool moves = start >= 0 && kept > j && (unsigned)from < (unsigned)a.pages && (unsigned)to < (unsigned)a.pages;
      from_at[0][tid] = moves ? from * a.k_b + from_off * a.k_l : -1;
      from_at[1][tid] = moves ? from * a.v_b + from_off * a.v_l : -1;
      to_at[0][tid] = moves ? to * a.k_b + to_off * a.k_l : -1;
      to_at[1][tid] = moves ? to * a.v_b + to_off * a.v_l : -1;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
    for (int i0 = 0; works && i0 < n; i0 += kAtOnce) {
      uintx4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) x[i] = *reinterpret_cast<const uintx4*>(rows + max(from_at[is_v][min(i0 + i, n - 1)], (int64_t)0));
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (i0 + i < n && to_at[is_v][i0 + i] >= 0) *reinterpret_cast<uintx4*>(rows + to_at[is_v][i0 + i]) = x[i];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
  }
}

// ---- sequences that go on from others --------------------------------------------------------------
// New sequence j shares the whole pages of its parent.  The page that is not full, if there is one, goes to the first new sequence of the parent; each
// further one gets the next of the free pages, and a copy of its tokens to make.  Every workgroup finds the first ones (a minimum, whatever the order of
// its parts) and the running sum of the pages for itself, then writes its rows.
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

// The first tokens of a page to the same places of another: a 16-byte chunk of K and of V to a lane, in the order of memory.
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
  const int items = (a.by_token ? tokens : a.page) * a.heads << a.chunk_bits;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < items; i += gridDim.y * 256) {
    const int row = i >> a.chunk_bits, outer = (int)a.inner.div(row), in = row - outer * (int)a.inner.d;
    const int64_t h = a.by_token ? in : outer, t = a.by_token ? outer : in, at = (i & ((1 << a.chunk_bits) - 1)) * 16;
    if (t >= tokens) continue;
    const uintx4 k = *reinterpret_cast<const uintx4*>(a.k + from * a.k_b + h * a.k_h + t * a.k_l + at);
    const uintx4 v = *reinterpret_cast<const uintx4*>(a.v + from * a.v_b + h * a.v_h + t * a.v_l + at);
    *reinterpret_cast<uintx4*>(a.k + to * a.k_b + h * a.k_h + t * a.k_l + at) = k;
    *reinterpret_cast<uintx4*>(a.v + to * a.v_b + h * a.v_h + t * a.v_l + at) = v;
  }
}

// ---- the pages that no one holds -------------------------------------------------------------------
// A bit for every page, set by the table rows as far as their lengths need pages; then the ids whose bit is not set, in order.
struct FreeArgs {
  const int32_t *table, *lens;
  int64_t table_stride;
  int n, row_tokens, pages, words;          // words of 32 bits
  int32_t *free_pages, *count;
  uint32_t* used;                           // workspace
  FastDiv page;
};
// Marks the pages of the row of a wave.
template <class Mark>
__device__ __forceinline__ void mark_row(const FreeArgs& a, int i, Mark mark) {
  const int held = pages_of(a.page, min(max(a.lens[i], 0), a.row_tokens));
  const int32_t* const row = a.table + (int64_t)i * a.table_stride;
  for (int p = threadIdx.x & 63; p < held; p += 64) {
    const int id = row[p];
    if ((unsigned)id < (unsigned)a.pages) mark(id);
  }
}
// The free pages of words [first, first + n) of `used` (the last word's bits past the end are set), by the whole workgroup, from place `at` of the list on.
template <int kThreads>
__device__ __forceinline__ int list_free(const FreeArgs& a, const uint32_t* used, int first, int n, int at, int* wave_sum) {
  constexpr int kGroupWaves = kThreads / 64;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int each = (n + kGroupWaves - 1) / kGroupWaves, w0 = min(wave * each, n), w1 = min(w0 + each, n);       // words of a wave
  int mine = 0;
  for (int w = w0 + lane; w < w1; w += 64) mine += __popc(~used[first + w]);
  const int sum = __builtin_amdgcn_readlane((int)wave_scan((uint32_t)mine, sum_of), 63);
  if (lane == 0) wave_sum[wave] = sum;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int all = at;
  for (int w = 0; w < kGroupWaves; ++w) {
    if (w < wave) at += wave_sum[w];
    all += wave_sum[w];
  }
  for (int w = w0; w < w1; w += 2) {           // 64 pages at a time
    const bool free = w + (lane >> 5) < w1 && !(used[first + min(w + (lane >> 5), w1 - 1)] >> (lane & 31) & 1);
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
  for (int w = threadIdx.x; w < a.words; w += 1024) used[w] = past_the_end(a, w);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  for (int i = threadIdx.x >> 6; i < a.n; i += 16) mark_row(a, i, [&](int id) { atomicOr(&used[id >> 5], 1u << (id & 31)); });
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int all = list_free<1024>(a, used, 0, a.words, 0, wave_sum);
  if (threadIdx.x == 0) *a.count = all;
}
__global__ __launch_bounds__(256) void free_clear_kernel(FreeArgs a) {
  const int w = blockIdx.x * 256 + threadIdx.x;
  if (w < a.words) a.used[w] = past_the_end(a, w);
}
__global__ __launch_bounds__(256) void free_mark_kernel(FreeArgs a) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i < a.n) mark_row(a, i, [&](int id) { atomicOr(&a.used[id >> 5], 1u << (id & 31)); });
}
__global__ __launch_bounds__(1024) void free_list_kernel(FreeArgs a, int words_each) {
  __shared__ int before[16], wave_sum[16];
  const int first = blockIdx.x * words_each, n = min(words_each, a.words - first), tid = threadIdx.x;
  int mine = 0;
  for (int w = tid; w < first; w += 1024) mine += __popc(~a.used[w]);
  const int sum = __builtin_amdgcn_readlane((int)wave_scan((uint32_t)mine, sum_of), 63);
  if ((tid & 63) == 0) before[tid >> 6] = sum;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int at = 0;
  for (int w = 0; w < 16; ++w) at += before[w];
  const int all = list_free<1024>(a, a.used, first, n, at, wave_sum);
  if (first + n == a.words && tid == 0) *a.count = all;
}
// In one workgroup, or in three launches over the device.
bool free_in_one(int n_seq, int width, int n_pages) { return n_pages <= (1 << 18) && (int64_t)n_seq * width <= (1 << 16); }

}  // namespace

basa_status launch_tree_masks(const int32_t* parents, const int32_t* cu, int n, int tokens, int64_t* masks, int words, int64_t mask_stride,
                              int32_t* depths, hipStream_t st) {
  if (n == 0) return BASA_OK;
  ProfScope prof(K_PAGED, st);
  tree_masks_kernel<<<n, 256, words * 64 * 12, st>>>(parents, cu, tokens, reinterpret_cast<uint64_t*>(masks), words, mask_stride, depths);
  BASA_HIP_CHECK_LAUNCH("tree_masks_kernel");
  return BASA_OK;
}

basa_status launch_cache_compact(const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width, int64_t table_stride,
                                 const int32_t* start, const int32_t* keep, int most, int64_t keep_stride, const int32_t* count, int n,
                                 hipStream_t st) {
  if (n == 0 || most == 0) return BASA_OK;
  CompactArgs a{};
  const int e = k_pages.dtype == BASA_BF16 ? 2 : 4;
  a.k = static_cast<char*>(const_cast<void*>(k_pages.ptr)); a.v = static_cast<char*>(const_cast<void*>(v_pages.ptr));
  a.k_b = k_pages.stride_b * e; a.k_h = k_pages.stride_h * e; a.k_l = k_pages.stride_l * e;
  a.v_b = v_pages.stride_b * e; a.v_h = v_pages.stride_h * e; a.v_l = v_pages.stride_l * e;
  a.table = table; a.start = start; a.keep = keep; a.count = count; a.table_stride = table_stride; a.keep_stride = keep_stride;
  a.width = width; a.most = most; a.pages = k_pages.batch;
  while ((16 << a.chunk_bits) < k_pages.d * e) ++a.chunk_bits;
  a.chunks = k_pages.heads << a.chunk_bits;
  a.page = fast_div((uint32_t)k_pages.L);
  ProfScope prof(K_PAGED, st);
  compact_kernel<<<dim3(n, ceil_div(2 * a.chunks, 256)), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("compact_kernel");
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
  return free_in_one(n_seq, width, n_pages) ? 256 : align_up((size_t)ceil_div(n_pages, 32) * 4, 256);
}
basa_status launch_page_free(const int32_t* table, int width, int64_t table_stride, const int32_t* lens, int n_seq, int page, int n_pages,
                             int32_t* free_pages, int32_t* count, void* ws, hipStream_t st) {
  FreeArgs a{};
  a.table = table; a.lens = lens; a.table_stride = table_stride; a.n = n_seq; a.row_tokens = width * page; a.pages = n_pages;
  a.words = ceil_div(n_pages, 32); a.free_pages = free_pages; a.count = count; a.used = static_cast<uint32_t*>(ws);
  a.page = fast_div((uint32_t)page);
  ProfScope prof(K_PAGED, st);
  if (free_in_one(n_seq, width, n_pages)) {
    page_free_kernel<<<1, 1024, std::max(a.words * 4, 16), st>>>(a);
    BASA_HIP_CHECK_LAUNCH("page_free_kernel");
    return BASA_OK;
  }
  free_clear_kernel<<<ceil_div(a.words, 256), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("free_clear_kernel");
  if (n_seq > 0) {
    free_mark_kernel<<<ceil_div(n_seq, 4), 256, 0, st>>>(a);
    BASA_HIP_CHECK_LAUNCH("free_mark_kernel");
  }
  const int groups = std::min(ceil_div(a.words, 64), 64), each = ceil_div(a.words, groups);
  free_list_kernel<<<ceil_div(a.words, each), 1024, 0, st>>>(a, each);
  BASA_HIP_CHECK_LAUNCH("free_list_kernel");
  return BASA_OK;
}

}  // namespace basa
