// Pages of a cache for new tokens and back: block tables, slots and positions from the lengths of the sequences, on the device.
//
// Who gets which page is a matter of two prefix sums over the sequences (rows, and pages), for which one workgroup walks them; the rows' slots then follow from the
// sequence's own numbers, for any number of workgroups.
#include "nat_internal.h"

namespace nat {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

struct PageArgs {
  int32_t* table;
  const int32_t *lens, *change, *counts;      // change: new tokens (reserve), or tokens that stay (release)
  int32_t* free_pages;
  int32_t *counts_out, *lens_out, *start, *cu, *pos;
  int64_t* slots;
  int32_t* ws;           // reserve: [n_seqs] place on the stack of a sequence's first new page;  release: [n_seqs] pages that go back, and n_free
  int32_t width, n_seqs, n_pages, page_log2;
  int64_t rows_cap;
};

__device__ __forceinline__ int clamped(int x, int64_t most) { return x < 0 ? 0 : x < most ? x : (int)most; }
__device__ __forceinline__ int64_t pages_of(int64_t tokens, int log2) { return (tokens + (1 << log2) - 1) >> log2; }

// Inclusive prefix sum over the workgroup; *all: of all threads
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* wave_sums, int64_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  int64_t before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? wave_sums[w] : 0;
    sum += wave_sums[w];
  }
  *all = sum;
  return before + x;
}

// Sequence by sequence: where its rows begin, whether it is served, which pages it gets
__device__ __forceinline__ void plan(const PageArgs& a, int64_t* wave_sums) {
  const int64_t most = (int64_t)a.width << a.page_log2;
  const int n_free = clamped(a.counts[0], a.n_pages);
  int64_t rows = 0, asked = 0, given = 0;
  int refused = 0;
  if (threadIdx.x == 0) a.cu[0] = 0;
  for (int first = 0; first < a.n_seqs; first += kThreads) {
    const int i = first + (int)threadIdx.x;
    const bool there = i < a.n_seqs;
    const int len = there ? clamped(a.lens[i], most) : 0, more = there && a.change[i] > 0 ? a.change[i] : 0;
    int64_t all;
    const int64_t end = rows + block_sum(more, wave_sums, &all);
    rows += all;
    bool served = len + (int64_t)more <= most && (more == 0 || end <= a.rows_cap);
    const int64_t need = served ? pages_of(len + (int64_t)more, a.page_log2) - pages_of(len, a.page_log2) : 0;
    const int64_t upto = asked + block_sum(need, wave_sums, &all);
    asked += all;
    served = served && (need == 0 || upto <= n_free);
    block_sum(served ? need : 0, wave_sums, &all);
    given += all;
    block_sum(there && !served, wave_sums, &all);
    refused += (int)all;
    if (there) {
      a.cu[i + 1] = end < INT32_MAX ? (int)end : INT32_MAX;
      a.start[i] = served ? len : -1;
      a.lens_out[i] = served ? len + more : len;
      a.ws[i] = (int)(n_free - 1 - (upto - need));      // (unused by those that get none)
    }
  }
  if (threadIdx.x == 0) {
    a.counts_out[0] = (int)(n_free - given);
    a.counts_out[1] = refused;
  }
}

// Slots, positions and the table's new entries, a row per thread
__device__ __forceinline__ void fill_row(const PageArgs& a, int64_t row) {
  int64_t slot = -1;
  int pos = 0;
  if (row < a.cu[a.n_seqs]) {
    const int seq = rollout_of_pos(a.cu, 0, a.n_seqs, row), start = a.start[seq];
    const int64_t most = (int64_t)a.width << a.page_log2;
    const int at = (int)(row - a.cu[seq]);
    const int64_t to = (int64_t)(start < 0 ? clamped(a.lens_out[seq], most) : start) + at;
    pos = to < INT32_MAX ? (int)to : INT32_MAX;              // (a refused sequence may ask for anything)
    if (start >= 0) {
      const int place = pos >> a.page_log2, fresh = (int)pages_of(start, a.page_log2);
      int page;
      if (place < fresh) {
        page = a.table[(int64_t)seq * a.width + place];
      } else {
        page = a.free_pages[a.ws[seq] - (place - fresh)];
        if (at == 0 || (pos & ((1 << a.page_log2) - 1)) == 0) a.table[(int64_t)seq * a.width + place] = page;
      }
      if (page >= 0 && page < a.n_pages) slot = ((int64_t)page << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
    }
  }
  a.slots[row] = slot;
  if (a.pos) a.pos[row] = pos;
}

__global__ void __launch_bounds__(kThreads) reserve_plan_kernel(PageArgs a) {
  __shared__ int64_t wave_sums[kWaves];
  plan(a, wave_sums);
}

__global__ void __launch_bounds__(256) reserve_fill_kernel(PageArgs a, int64_t first) {
  const int64_t row = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row < a.rows_cap) fill_row(a, row);
}

// ------------------------------------------------------------------ back ----
constexpr int kDirectSeqs = 4096;                // up to so many sequences, each adds up the counts of those before it by itself
struct Back { int kept, from, to; };             // tokens that stay; places whose pages go back
__device__ __forceinline__ Back back_of(const PageArgs& a, int seq) {
  const int64_t most = (int64_t)a.width << a.page_log2;
  const int len = clamped(a.lens[seq], most), kept = clamped(a.change[seq], len);
  return {kept, (int)pages_of(kept, a.page_log2), (int)pages_of(len, a.page_log2)};
}
__device__ __forceinline__ bool goes_back(const PageArgs& a, int seq, int place, int* page) {
  *page = a.table[(int64_t)seq * a.width + place];
  return *page >= 0 && *page < a.n_pages;
}

// A wavefront per sequence counts
__global__ void __launch_bounds__(256) release_count_kernel(PageArgs a) {
  const int lane = threadIdx.x & 63, seq = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.ws[a.n_seqs] = clamped(a.counts[0], a.n_pages);
  if (seq >= a.n_seqs) return;
  const Back b = back_of(a, seq);
  int n = 0, page;
  for (int place = b.from + lane; place < b.to; place += 64) n += goes_back(a, seq, place, &page);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d, 64);
  if (lane == 0) a.ws[seq] = n;
}

// of many sequences: the pages of those before each
__global__ void __launch_bounds__(kThreads) release_scan_kernel(PageArgs a) {
  __shared__ int64_t wave_sums[kWaves];
  int64_t before = 0;
  for (int first = 0; first < a.n_seqs; first += kThreads) {
    const int i = first + (int)threadIdx.x, n = i < a.n_seqs ? a.ws[i] : 0;
    int64_t all;
    const int64_t to = before + block_sum(n, wave_sums, &all) - n;
    if (i < a.n_seqs) a.ws[i] = to < INT32_MAX ? (int)to : INT32_MAX;
    before += all;
  }
}

// and puts them where those of the sequences before it end
template <bool kScanned>
__global__ void __launch_bounds__(256) release_fill_kernel(PageArgs a) {
  const int lane = threadIdx.x & 63, seq = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (seq >= a.n_seqs) return;
  const Back b = back_of(a, seq);
  int64_t to = 0;
  if constexpr (kScanned) {
    to = a.ws[seq];
  } else {
    for (int i = lane; i < seq; i += 64) to += a.ws[i];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) to += __shfl_xor(to, d, 64);
  }
  to += a.ws[a.n_seqs];
  for (int first = b.from; first < b.to; first += 64) {
    const int place = first + lane;
    int page = -1;
    const bool back = place < b.to && goes_back(a, seq, place, &page);
    const uint64_t with = __ballot(back);
    const int64_t at = to + __popcll(with & ((uint64_t{1} << lane) - 1));
    if (back && at < a.n_pages) a.free_pages[at] = page;
    to += __popcll(with);
  }
  if (lane == 0) {
    a.lens_out[seq] = b.kept;
    if (seq == a.n_seqs - 1) {
      a.counts_out[0] = to < a.n_pages ? (int)to : a.n_pages;
      a.counts_out[1] = 0;
    }
  }
}

__global__ void pages_nothing_kernel(PageArgs a) {
  if (a.cu) a.cu[0] = 0;
  a.counts_out[0] = clamped(a.counts[0], a.n_pages);
  a.counts_out[1] = 0;
}

nat_status page_args(const int32_t* d_block_table, int32_t width, int32_t n_seqs, int32_t page_size, const int32_t* d_lens, const int32_t* d_change,
                     const int32_t* d_free_pages, int32_t n_pages, const int32_t* d_counts, int32_t* d_counts_out, int32_t* d_lens_out, PageArgs* a) {
  if (n_seqs < 0 || width < 0 || n_pages < 0) return NAT_INVALID_ARG;
  int log2 = 4;
  while (log2 < 8 && (1 << log2) != page_size) ++log2;
  if ((1 << log2) != page_size || n_seqs > (1 << 24) || (int64_t)width << log2 > INT32_MAX) return NAT_BAD_SHAPE;
  if (!d_counts || !d_counts_out || (n_pages > 0 && !d_free_pages)) return NAT_INVALID_ARG;
  if (n_seqs > 0 && (!d_lens || !d_change || !d_lens_out || (width > 0 && !d_block_table))) return NAT_INVALID_ARG;
  *a = PageArgs{};
  a->table = (int32_t*)d_block_table;
  a->lens = d_lens;
  a->change = d_change;
  a->counts = d_counts;
  a->free_pages = (int32_t*)d_free_pages;
  a->counts_out = d_counts_out;
  a->lens_out = d_lens_out;
  a->width = width;
  a->n_seqs = n_seqs;
  a->n_pages = n_pages;
  a->page_log2 = log2;
  return NAT_OK;
}

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" size_t nat_kv_reserve_workspace_bytes(int32_t n_seqs) { return n_seqs <= 0 || n_seqs > (1 << 24) ? 0 : whole((size_t)n_seqs * 4); }

extern "C" nat_status nat_kv_reserve(int32_t* d_block_table, int32_t table_width, int32_t n_seqs, int32_t page_size, const int32_t* d_seq_lens,
                                     const int32_t* d_new_lens, const int32_t* d_free_pages, int32_t n_pages, const int32_t* d_counts, int64_t rows_cap,
                                     int32_t* d_counts_out, int32_t* d_seq_lens_out, int32_t* d_start, int32_t* d_cu_new, int64_t* d_slots,
                                     int32_t* d_position_ids, void* d_ws, size_t ws_bytes, void* stream) {
  PageArgs a;
  if (rows_cap < 0 || rows_cap > INT32_MAX) return NAT_INVALID_ARG;
  const nat_status st = page_args(d_block_table, table_width, n_seqs, page_size, d_seq_lens, d_new_lens, d_free_pages, n_pages, d_counts, d_counts_out,
                                  d_seq_lens_out, &a);
  if (st != NAT_OK) return st;
  if (!d_cu_new || (n_seqs > 0 && !d_start) || (rows_cap > 0 && !d_slots)) return NAT_INVALID_ARG;
  if (n_seqs > 0 && (!d_ws || ws_bytes < nat_kv_reserve_workspace_bytes(n_seqs))) return NAT_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)d_ws & 255) return NAT_INVALID_ARG;
  a.start = d_start;
  a.cu = d_cu_new;
  a.slots = d_slots;
  a.pos = d_position_ids;
  a.ws = (int32_t*)d_ws;
  a.rows_cap = rows_cap;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_PAGES, s);
  if (n_seqs > 0) reserve_plan_kernel<<<1, kThreads, 0, s>>>(a);
  else pages_nothing_kernel<<<1, 1, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  if (rows_cap == 0) return NAT_OK;
  reserve_fill_kernel<<<(unsigned)((rows_cap + 255) / 256), 256, 0, s>>>(a, 0);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}

extern "C" size_t nat_kv_release_workspace_bytes(int32_t n_seqs) { return n_seqs <= 0 || n_seqs > (1 << 24) ? 0 : whole(((size_t)n_seqs + 1) * 4); }

extern "C" nat_status nat_kv_release(const int32_t* d_block_table, int32_t table_width, int32_t n_seqs, int32_t page_size, const int32_t* d_seq_lens,
                                     const int32_t* d_keep_lens, int32_t* d_free_pages, int32_t n_pages, const int32_t* d_counts, int32_t* d_counts_out,
                                     int32_t* d_seq_lens_out, void* d_ws, size_t ws_bytes, void* stream) {
  PageArgs a;
  const nat_status st = page_args(d_block_table, table_width, n_seqs, page_size, d_seq_lens, d_keep_lens, d_free_pages, n_pages, d_counts, d_counts_out,
                                  d_seq_lens_out, &a);
  if (st != NAT_OK) return st;
  if (n_seqs > 0 && (!d_ws || ws_bytes < nat_kv_release_workspace_bytes(n_seqs))) return NAT_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)d_ws & 255) return NAT_INVALID_ARG;
  a.ws = (int32_t*)d_ws;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_PAGES, s);
  if (n_seqs > 0) {
    release_count_kernel<<<(n_seqs + 3) / 4, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
    if (n_seqs <= kDirectSeqs) {
      release_fill_kernel<false><<<(n_seqs + 3) / 4, 256, 0, s>>>(a);
    } else {
      release_scan_kernel<<<1, kThreads, 0, s>>>(a);
      NAT_LAUNCH_CHECK();
      release_fill_kernel<true><<<(n_seqs + 3) / 4, 256, 0, s>>>(a);
    }
  } else {
    pages_nothing_kernel<<<1, 1, 0, s>>>(a);
  }
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
