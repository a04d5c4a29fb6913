// The paged key-value cache: block tables and slot maps from request lengths, and rows moved into the pages and out of them.
#include <algorithm>
#include <climits>
#include "common.hpp"
#include "paged_plan.hpp"

namespace basa {
namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// Sums that stop at 2^32 - 1: those of the lengths may pass it, and what lies beyond 2^31 fits nowhere.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
// Running sum over the threads of a workgroup of 256: the sum of the values of all threads before this one; *all: of every thread.  An array
// serves one call.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* all, uint32_t (&wave_sum)[4]) {
  constexpr int kWaveShr1 = 0x138;
  const int wave = threadIdx.x >> 6;
  const uint32_t upto = wave_scan(v, add_sat);
  if ((threadIdx.x & 63) == 63) wave_sum[wave] = upto;
  uint32_t before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)upto, kWaveShr1, 0xf, 0xf, false);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t sum = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w == wave) before = add_sat(before, sum);
    sum = add_sat(sum, wave_sum[w]);
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
// Bound by latency: a step of 600 sequences reads and writes some 100 KB.  One launch without a hand-over between workgroups: every
// workgroup forms both running sums for itself (two words per sequence from the L2) and keeps them in the LDS, where its tokens look
// their sequence up.  The token that opens a page writes the page's table entry.  8 sequences, 8 tokens: 2.8 us; 40 sequences, 85000 tokens
// 5.3; 600 sequences, 15000 tokens 7.2; a step of 2000 sequences 9.0, of 8192 37, most of it the rounds of 256 lengths that are loaded one
// after the other; a kernel that does nothing 2.5.
struct PageTableArgs {
  const int32_t *have, *add, *free_pages;
  int32_t *table, *lens, *cu, *pages;
  int64_t* slots;
  int64_t table_stride;
  int n, n_free, tokens, tokens_per_group, row_tokens;
  FastDiv page;
};
constexpr int kMaxPagedSeqs = 8192;         // 96 KB of LDS
__device__ __forceinline__ int pages_of(const FastDiv& page, int tokens) {
  const int whole = (int)page.div(tokens);
  return whole + (whole * (int)page.d != tokens);
}

__global__ __launch_bounds__(256) void page_tables_kernel(PageTableArgs a) {
  extern __shared__ uint32_t words[];
  __shared__ uint32_t add_sum[4], need_sum[4];
  __shared__ int given;
  uint32_t* start = words;                  // new tokens of a sequence; then its first token in the slot map
  int32_t* have = reinterpret_cast<int32_t*>(words) + a.n;
  int32_t* first = have + a.n;              // pages it needs, -1: does not fit; then its place among the free pages, -1: not served
  const int tid = threadIdx.x, each = (a.n + 255) / 256;
  const int i0 = min(tid * each, a.n), i1 = min(i0 + each, a.n);
  if (tid == 0) given = 0;
  for (int i = tid; i < a.n; i += 256) {
    start[i] = max(a.add[i], 0);
    have[i] = max(a.have[i], 0);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t sum = 0, total, asked;
  for (int i = i0; i < i1; ++i) sum = add_sat(sum, start[i]);
  uint32_t at = sum_before(sum, &total, add_sum);
  sum = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t add = start[i], after = have[i] + add;             // (below 2^32)
    start[i] = at;
    at = add_sat(at, add);
    const bool fits = after <= (uint32_t)a.row_tokens && at <= (uint32_t)a.tokens;
    const int need = fits ? pages_of(a.page, (int)after) - pages_of(a.page, have[i]) : -1;
    first[i] = need;
    sum = add_sat(sum, (uint32_t)max(need, 0));
  }
  at = sum_before(sum, &asked, need_sum);
  int last = 0;
  for (int i = i0; i < i1; ++i) {
    const int need = first[i];
    if (need < 0) continue;
    const uint32_t end = add_sat(at, (uint32_t)need);
    const bool served = end <= (uint32_t)a.n_free;
    first[i] = served ? (int)at : -1;
    at = end;
    if (served) last = (int)end;
  }
  if (last > 0) atomicMax(&given, last);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  const int all = (int)min(total, (uint32_t)INT_MAX);
  for (int i = blockIdx.x * 256 + tid; i < a.n; i += gridDim.x * 256) {
    a.lens[i] = first[i] >= 0 ? have[i] + (int)((i + 1 < a.n ? start[i + 1] : total) - start[i]) : have[i];
    a.cu[i] = (int)min(start[i], (uint32_t)INT_MAX);
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.cu[a.n] = all;
    a.pages[0] = given;
    a.pages[1] = (int)min(asked, (uint32_t)INT_MAX);
  }
  const int t0 = blockIdx.x * a.tokens_per_group, t1 = min(a.tokens - t0, a.tokens_per_group) + t0;
  for (int t = t0 + tid; t < t1; t += 256) {
    int64_t slot = -1;
    if (t < all) {
      int lo = 0, hi = a.n;                 // the last sequence that starts at or before t: start[lo] <= t < start[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= (uint32_t)t) lo = mid; else hi = mid;
      }
      const int place = first[lo];
      if (place >= 0) {
        const int pos = have[lo] + (t - (int)start[lo]);
        const int p = (int)a.page.div(pos), off = pos - p * (int)a.page.d, held = pages_of(a.page, have[lo]);
        int32_t* entry = a.table + (int64_t)lo * a.table_stride + p;
        const int32_t* from = p >= held ? a.free_pages + place + p - held : entry;
        const int id = *from;
        if (p >= held && off == 0) *entry = id;
        if (id >= 0) slot = (int64_t)id * a.page.d + off;
      }
    }
    a.slots[t] = slot;
  }
}

// ---- rows into the pages and out of them -----------------------------------------------------------
// Packed rows [T][heads][d] on one side, pages [pages][heads][page][d] on the other, both with free strides.  Bound by the memory: each
// byte is read once and written once (41K tokens of 8 heads, 351 MB both ways: 66 us, 5.3 TB/s; a copy 5.2).  A workgroup takes a run of tokens: first one lane per token finds where the token lives (its
// slot, or its sequence and table entry), then the lanes copy 16-byte chunks, one of K and one of V each.  (Four chunks
// a lane, requested at once, in workgroups of eight times the tokens -> one: 655 MB gathered 252 -> 226 us, 41K tokens appended 73 -> 70.)
//
// Loads and stores through the caches or past them (bytes of K and V on one side; both sides are in the caches or not in turn as in a program
// that goes on to other tensors): rows that are appended are not read soon, streaming stores 3000 to 60000 tokens, 8 heads of 128 (12 to
// 246 MB): 6.3 -> 4.0, 15.4 -> 13.8, 35 -> 26, 98 -> 90 us.  Streaming loads pay from 128 MB on: 12 MB 4.0 -> 7.1, 82 MB 26 -> 30, 246 MB
// 90 -> 87; gathered, 82 MB 27.8 -> 29.5, 134 MB level, 174 MB 70 -> 59, 246 MB 90 -> 74.  What is gathered is read next and stays in
// the caches as long as they can hold it: stores past them 174 MB 59 -> 62, 246 MB 74 -> 85, 383 MB 134 -> 129, 655 MB 221 -> 211.
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
constexpr int kMaxRowTokens = 256, kRowChunks = 256;
constexpr int64_t kStreamLoadBytes = 128 << 20, kStreamStoreBytes = 256 << 20;
constexpr int64_t kSkip = -1, kZeros = -2;

template <bool kStream>
__device__ __forceinline__ uintx4 load_chunk(const char* at) {
  if constexpr (kStream) return __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(at));
  return *reinterpret_cast<const uintx4*>(at);
}
template <bool kStream>
__device__ __forceinline__ void store_chunk(char* at, uintx4 v) {
  if constexpr (kStream) __builtin_nontemporal_store(v, reinterpret_cast<uintx4*>(at));
  else *reinterpret_cast<uintx4*>(at) = v;
}

template <bool kGather, bool kStreamLoad, bool kStreamStore>
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
  for (int i = threadIdx.x; i < items; i += 256) {
    const int t = (int)a.row_chunks.div(i), rest = i - t * (int)a.row_chunks.d;
    const int64_t h = rest >> a.chunk_bits, c = (rest & mask) * 16, where = k_at[t];
    char* k_page = a.k_pages + max(where, (int64_t)0) + h * a.k_page_h + c;
    char* v_page = a.v_pages + max(v_at[t], (int64_t)0) + h * a.v_page_h + c;
    char* k_row = a.k_rows + (t0 + t) * a.k_row_t + h * a.k_row_h + c;
    char* v_row = a.v_rows + (t0 + t) * a.v_row_t + h * a.v_row_h + c;
    uintx4 k = load_chunk<kStreamLoad>(kGather ? k_page : k_row), v = load_chunk<kStreamLoad>(kGather ? v_page : v_row);
    if (where == kSkip) continue;
    if (kGather && where == kZeros) {
      k = uintx4{0u, 0u, 0u, 0u};
      v = uintx4{0u, 0u, 0u, 0u};
    }
    store_chunk<kStreamStore>(kGather ? k_row : k_page, k);
    store_chunk<kStreamStore>(kGather ? v_row : v_page, v);
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
  // a chunk of K and of V to a thread, fewer tokens where the device would not be full
  const int most = std::min(std::max(kRowChunks / (int)a.row_chunks.d, 1), kMaxRowTokens);
  // (and no more than 2^23 workgroups, 2^31 threads)
  a.tokens_per_group = std::max({1, std::min(most, ceil_div(a.T, 1024)), ceil_div(a.T, 1 << 23)});
  return a;
}
int64_t rows_bytes(const TensorView& k) { return (int64_t)2 * k.L * k.heads * k.d * (k.dtype == BASA_BF16 ? 2 : 4); }

}  // namespace

bool page_tables_take(int n_seq) { return n_seq <= kMaxPagedSeqs; }

basa_status launch_page_tables(const int32_t* have, const int32_t* add, int n, int page, int32_t* table, int width, int64_t table_stride,
                               const int32_t* free_pages, int n_free, int64_t* slots, int tokens, int32_t* lens, int32_t* cu,
                               int32_t* pages, hipStream_t st) {
  PageTableArgs a{};
  a.have = have; a.add = add; a.free_pages = free_pages; a.table = table; a.lens = lens; a.cu = cu; a.pages = pages; a.slots = slots;
  a.table_stride = table_stride; a.n = n; a.n_free = n_free; a.tokens = tokens; a.row_tokens = width * page;
  a.page = fast_div((uint32_t)page);
  a.tokens_per_group = std::max(256, ceil_div(tokens, 1024));
  const int groups = std::max(ceil_div(tokens, a.tokens_per_group), 1);
  const int lds = std::max(n * 12, 16);
  if (lds > 60 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&page_tables_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(dynamic LDS)");
  }
  ProfScope prof(K_PAGED, st);
  page_tables_kernel<<<groups, 256, lds, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("page_tables_kernel");
  return BASA_OK;
}

basa_status launch_cache_append(const TensorView& k, const TensorView& v, const int64_t* slots, const TensorView& k_pages,
                                const TensorView& v_pages, hipStream_t st) {
  RowsArgs a = rows_args(k, v, k_pages, v_pages);
  a.slots = slots;
  ProfScope prof(K_PAGED, st);
  const int groups = ceil_div(a.T, a.tokens_per_group);
  if (rows_bytes(k) < kStreamLoadBytes) cache_rows_kernel<false, false, true><<<groups, 256, 0, st>>>(a);
  else cache_rows_kernel<false, true, true><<<groups, 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("cache_rows_kernel");
  return BASA_OK;
}

basa_status launch_cache_gather(const TensorView& k_pages, const TensorView& v_pages, const int32_t* table, int width,
                                int64_t table_stride, const int32_t* cu, int n, const TensorView& k, const TensorView& v, hipStream_t st) {
  RowsArgs a = rows_args(k, v, k_pages, v_pages);
  a.table = table; a.width = width; a.table_stride = table_stride; a.cu = cu; a.n = n;
  ProfScope prof(K_PAGED, st);
  const int groups = ceil_div(a.T, a.tokens_per_group);
  const int64_t bytes = rows_bytes(k);
  if (bytes < kStreamLoadBytes) cache_rows_kernel<true, false, false><<<groups, 256, 0, st>>>(a);
  else if (bytes <= kStreamStoreBytes) cache_rows_kernel<true, true, false><<<groups, 256, 0, st>>>(a);
  else cache_rows_kernel<true, true, true><<<groups, 256, 0, st>>>(a);
  BASA_HIP_CHECK_LAUNCH("cache_rows_kernel");
  return BASA_OK;
}

}  // namespace basa
