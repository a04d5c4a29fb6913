// The paged key-value cache: block tables and slot maps from request lengths, and rows moved into the pages and out of them.
#include <algorithm>
#include <climits>
#include "common.hpp"
#include "paged_plan.hpp"

namespace basa {
namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// Running sum over the threads of a workgroup of 256: the sum of the values of all threads before this one; *all: of every thread.  An array
// serves one call.
__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t* all, int64_t (&wave_sum)[4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) wave_sum[wave] = x;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int64_t before = x - v, sum = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += wave_sum[w];
    sum += wave_sum[w];
  }
  *all = sum;
  return before;
}

// ---- block tables and slot maps -------------------------------------------------------------------
// c_i = sum of add_j, j < i; a sequence fits if have + add tokens fit its table row and its tokens fit the slot map; it needs
// ceil((have + add) / page) - ceil(have / page) pages if it fits and 0 otherwise, and gets them from place f_i = sum of need_j, j < i, of
// the free pages on if there are that many.  (Behind the first sequence that is short of pages every other that needs one is short
// too, so that the pages given out are the first ones.)  Two running sums over the sequences, then one independent slot per token.
//
// Bound by latency: a step of 600 sequences reads and writes 70 KB.  One launch without a hand-over between workgroups: every
// workgroup forms both running sums for itself (two words per sequence from the L2) and keeps them in the LDS, where its tokens look
// their sequence up.  The token that opens a page writes the page's table entry.
struct PageTableArgs {
  const int32_t *have, *add, *free_pages;
  int32_t *table, *lens, *cu, *pages;
  int64_t* slots;
  int64_t table_stride;
  int n, n_free, tokens, tokens_per_group, row_tokens;
  FastDiv page;
};
constexpr int kMaxPagedSeqs = 8192;         // 64 KB of LDS for the two sums
__device__ __forceinline__ int pages_of(const FastDiv& page, int tokens) {
  const int whole = (int)page.div(tokens);
  return whole + (whole * (int)page.d != tokens);
}

__global__ __launch_bounds__(256) void page_tables_kernel(PageTableArgs a) {
  extern __shared__ int32_t sums[];
  __shared__ int64_t add_sum[4], need_sum[4];
  __shared__ int given;
  int32_t* start = sums;                    // first token of a sequence in the slot map (cut at 2^31 - 1)
  int32_t* first = sums + a.n;              // its place among the free pages, -1: not served
  const int tid = threadIdx.x, each = (a.n + 255) / 256;
  const int i0 = min(tid * each, a.n), i1 = min(i0 + each, a.n);
  if (tid == 0) given = 0;
  int64_t sum = 0, total, asked;
  for (int i = i0; i < i1; ++i) sum += max(a.add[i], 0);
  int64_t at = sum_before(sum, &total, add_sum);
  sum = 0;
  for (int i = i0; i < i1; ++i) {
    const int add = max(a.add[i], 0), have = max(a.have[i], 0);
    const bool fits = (int64_t)have + add <= a.row_tokens && at + add <= a.tokens;
    // (both counts are below 2^31 where it fits)
    const int need = fits ? pages_of(a.page, have + add) - pages_of(a.page, have) : -1;
    start[i] = (int)min(at, (int64_t)INT_MAX);
    first[i] = need;
    at += add;
    sum += max(need, 0);
  }
  at = sum_before(sum, &asked, need_sum);
  int last = 0;
  for (int i = i0; i < i1; ++i) {
    const int need = first[i];
    if (need < 0) continue;
    const bool served = at + need <= a.n_free;
    first[i] = served ? (int)at : -1;
    at += need;
    if (served) last = (int)at;
  }
  if (last > 0) atomicMax(&given, last);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int all = (int)min(total, (int64_t)INT_MAX);
  for (int i = blockIdx.x * 256 + tid; i < a.n; i += gridDim.x * 256) {
    const int have = max(a.have[i], 0), add = max(a.add[i], 0);
    a.lens[i] = first[i] >= 0 ? have + add : have;
    a.cu[i] = start[i];
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.cu[a.n] = all;
    a.pages[0] = given;
    a.pages[1] = (int)min(asked, (int64_t)INT_MAX);
  }
  const int t0 = blockIdx.x * a.tokens_per_group, t1 = min(a.tokens - t0, a.tokens_per_group) + t0;
  for (int t = t0 + tid; t < t1; t += 256) {
    int64_t slot = -1;
    if (t < all) {
      int lo = 0, hi = a.n;                 // the last sequence that starts at or before t: start[lo] <= t < start[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= t) lo = mid; else hi = mid;
      }
      const int place = first[lo];
      if (place >= 0) {
        const int have = max(a.have[lo], 0), pos = have + (t - start[lo]);
        const int p = (int)a.page.div(pos), off = pos - p * (int)a.page.d;
        const int held = pages_of(a.page, have);
        int32_t* entry = a.table + (int64_t)lo * a.table_stride + p;
        int id;
        if (p >= held) {
          id = a.free_pages[place + p - held];
          if (off == 0) *entry = id;
        } else {
          id = *entry;
        }
        if (id >= 0) slot = (int64_t)id * a.page.d + off;
      }
    }
    a.slots[t] = slot;
  }
}

// ---- rows into the pages and out of them -----------------------------------------------------------
// Packed rows [T][heads][d] on one side, pages [pages][heads][page][d] on the other, both with free strides.  Bound by the memory: each
// byte is read once and written once.  A workgroup takes a run of tokens: first one lane per token finds where the token lives (its
// slot, or its sequence and table entry), then all lanes copy 16-byte chunks of K and V, several requested before the first is stored.
struct RowsArgs {
  char *k_rows, *v_rows;                    // packed, bytes; strides of a token and of a head
  int64_t k_row_t, k_row_h, v_row_t, v_row_h;
  char *k_pages, *v_pages;
  int64_t k_page_b, k_page_h, k_page_l, v_page_b, v_page_h, v_page_l;
  const int64_t* slots;                     // append
  const int32_t *table, *cu;                // gather
  int64_t table_stride;
  int n, width, T, tokens_per_group, pages, chunk_bits;
  FastDiv page, row_chunks;                 // 16-byte chunks of one token: heads << chunk_bits
};
constexpr int kMaxRowTokens = 256, kRowsAtOnce = 4;
constexpr int64_t kSkip = -1, kZeros = -2;

template <bool kGather>
__global__ __launch_bounds__(256) void cache_rows_kernel(RowsArgs a) {
  __shared__ int64_t k_at[kMaxRowTokens], v_at[kMaxRowTokens];
  const int t0 = blockIdx.x * a.tokens_per_group, count = min(a.T - t0, a.tokens_per_group);
  if ((int)threadIdx.x < count) {
    const int t = t0 + threadIdx.x;
    int64_t id = -1, off = 0, none = kSkip;
    if constexpr (kGather) {
      if (t >= a.cu[0] && t < a.cu[a.n]) {
        int lo = 0, hi = a.n;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (a.cu[mid] <= t) lo = mid; else hi = mid;
        }
        const int64_t pos = (int64_t)t - a.cu[lo];
        none = kZeros;
        if (pos >= 0 && pos <= INT_MAX) {
          const int p = (int)a.page.div((uint32_t)pos);
          off = pos - (int64_t)p * a.page.d;
          if (p < a.width) id = a.table[(int64_t)lo * a.table_stride + p];
        }
      }
    } else {
      const int64_t slot = a.slots[t];
      if (slot >= 0) {
        id = slot <= INT_MAX ? (int64_t)a.page.div((uint32_t)slot) : slot / a.page.d;
        off = slot - id * a.page.d;
      }
    }
    const bool valid = id >= 0 && id < a.pages;
    k_at[threadIdx.x] = valid ? id * a.k_page_b + off * a.k_page_l : none;
    v_at[threadIdx.x] = valid ? id * a.v_page_b + off * a.v_page_l : none;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int items = count * (int)a.row_chunks.d, mask = (1 << a.chunk_bits) - 1;
  for (int i0 = threadIdx.x; i0 < items; i0 += 256 * kRowsAtOnce) {
    uintx4 kv[kRowsAtOnce], vv[kRowsAtOnce];
    int64_t k_to[kRowsAtOnce], v_to[kRowsAtOnce], where[kRowsAtOnce];
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      const int i = min(i0 + u * 256, items - 1);
      const int t = (int)a.row_chunks.div(i), rest = i - t * (int)a.row_chunks.d;
      const int64_t h = rest >> a.chunk_bits, c = (rest & mask) * 16;
      where[u] = k_at[t];
      const int64_t k_page = max(where[u], (int64_t)0) + h * a.k_page_h + c, v_page = max(v_at[t], (int64_t)0) + h * a.v_page_h + c;
      const int64_t k_row = (t0 + t) * a.k_row_t + h * a.k_row_h + c, v_row = (t0 + t) * a.v_row_t + h * a.v_row_h + c;
      k_to[u] = kGather ? k_row : k_page;
      v_to[u] = kGather ? v_row : v_page;
      kv[u] = *reinterpret_cast<const uintx4*>(kGather ? a.k_pages + k_page : a.k_rows + k_row);
      vv[u] = *reinterpret_cast<const uintx4*>(kGather ? a.v_pages + v_page : a.v_rows + v_row);
    }
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      if (i0 + u * 256 >= items || where[u] == kSkip) continue;
      if (kGather && where[u] == kZeros) {
        kv[u] = uintx4{0u, 0u, 0u, 0u};
        vv[u] = uintx4{0u, 0u, 0u, 0u};
      }
      *reinterpret_cast<uintx4*>((kGather ? a.k_rows : a.k_pages) + k_to[u]) = kv[u];
      *reinterpret_cast<uintx4*>((kGather ? a.v_rows : a.v_pages) + v_to[u]) = vv[u];
    }
  }
}

RowsArgs rows_args(const TensorView& k, const TensorView& v, const TensorView& k_pages, const TensorView& v_pages) {
  RowsArgs a{};
  const int e = k.dtype == BASA_BF16 ? 2 : 4;
  auto bytes = [](const void* p) { return const_cast<char*>(static_cast<const char*>(p)); };
  a.k_rows = bytes(k.ptr); a.v_rows = bytes(v.ptr);
  a.k_row_t = k.stride_l * e; a.k_row_h = k.stride_h * e; a.v_row_t = v.stride_l * e; a.v_row_h = v.stride_h * e;
  a.k_pages = bytes(k_pages.ptr); a.v_pages = bytes(v_pages.ptr);
  a.k_page_b = k_pages.stride_b * e; a.k_page_h = k_pages.stride_h * e; a.k_page_l = k_pages.stride_l * e;
  a.v_page_b = v_pages.stride_b * e; a.v_page_h = v_pages.stride_h * e; a.v_page_l = v_pages.stride_l * e;
  a.T = k.L; a.pages = k_pages.batch;
  a.page = fast_div((uint32_t)k_pages.L);
  while ((16 << a.chunk_bits) < k.d * e) ++a.chunk_bits;
  a.row_chunks = fast_div((uint32_t)k.heads << a.chunk_bits);
  // about eight chunks of K and of V to a thread, fewer where the device would not be full
  const int most = std::min(std::max(2048 / (int)a.row_chunks.d, 1), kMaxRowTokens);
  a.tokens_per_group = std::max(1, std::min(most, ceil_div(a.T, 1024)));
  return a;
}

}  // namespace

bool page_tables_take(int n_seq) { return n_seq <= kMaxPagedSeqs; }

basa_status launch_page_tables(const int32_t* have, const int32_t* add, int n, int page, int32_t* table, int width, int64_t table_stride,
                               const int32_t* free_pages, int n_free, int64_t* slots, int tokens, int32_t* lens, int32_t* cu,
                               int32_t* pages, hipStream_t st) {
  PageTableArgs a{};
  a.have = have; a.add = add; a.free_pages = free_pages; a.table = table; a.lens = lens; a.cu = cu; a.pages = pages; a.slots = slots;
  a.table_stride = table_stride; a.n = n; a.n_free = n_free; a.tokens = tokens; a.row_tokens = width * page;
  a.page = fast_div((uint32_t)page);
  const int groups = std::min(std::max(ceil_div(tokens, 1024), 1), 1024);
  a.tokens_per_group = ceil_div(tokens, groups);
  ProfScope prof(K_PAGED, st);
  page_tables_kernel<<<groups, 256, std::max((size_t)n * 8, (size_t)16), st>>>(a);
  BASA_HIP_CHECK_LAUNCH("page_tables_kernel");
  return BASA_OK;
}

basa_status launch_cache_append(const TensorView& k, const TensorView& v, const int64_t* slots, const TensorView& k_pages,
                                const TensorView& v_pages, hipStream_t st) {
  RowsArgs a = rows_args(k, v, k_pages, v_pages);
  a.slots = slots;
  ProfScope prof(K_PAGED, st);
  cache_rows_kernel<false><<<ceil_div(a.T, a.tokens_per_group), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("cache_rows_kernel");
  return BASA_OK;
}

basa_status launch_cache_gather(const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width,
                                int64_t table_stride, const int32_t* cu, int n, const TensorView& k, const TensorView& v, hipStream_t st) {
  RowsArgs a = rows_args(k, v, k_pages, v_pages);
  a.table = table; a.width = width; a.table_stride = table_stride; a.cu = cu; a.n = n;
  ProfScope prof(K_PAGED, st);
  cache_rows_kernel<true><<<ceil_div(a.T, a.tokens_per_group), 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("cache_rows_kernel");
  return BASA_OK;
}

}  // namespace basa
