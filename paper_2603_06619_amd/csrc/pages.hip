// Pages of a cache for new tokens and back: block tables, slots and positions from the lengths of the sequences, on the device.
//
// Who gets which page is a matter of two prefix sums over the sequences (rows, and pages), for which one workgroup walks them; the rows' slots then follow from the
// sequence's own numbers, for any number of workgroups.  Latency: a step of 512 sequences 4.5 us, a batch of 192 with 162 thousand new rows 5.6, its release 3.7 + 4.9.
#include "nat_internal.h"

#include <type_traits>

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

// Sums of numbers that are not negative, at most 2^32 - 1: in any order the same
__device__ __forceinline__ uint32_t add(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// Inclusive prefix sum over the wavefront, and over the workgroup: *all of all threads.  One barrier: `sums` may be used again behind the next one.
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  auto from = [](uint32_t v, auto ctrl, auto rows) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
  };
  using std::integral_constant;
  x = add(x, from(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{}));      // 1, 2, 4, 8 lanes on, inside rows of 16
  x = add(x, from(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{}));
  x = add(x, from(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{}));
  x = add(x, from(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{}));
  x = add(x, from(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));      // the last of a row to the next one, of two rows to the next two
  x = add(x, from(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));
  return x;
}
__device__ __forceinline__ uint32_t block_sum(uint32_t x, uint32_t* sums, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_sum(x);
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before = add(before, w < wave ? sums[w] : 0);
    total = add(total, sums[w]);
  }
  *all = total;
  return add(before, x);
}

// What a sequence's rows are made from
struct Served { int32_t *cu, *start, *len, *top; };      // offsets; first position, -1: refused; length afterwards; place on the stack of the first new page

// Sequence by sequence: where its rows begin, whether it is served, which pages it gets.  The results go to the caller's arrays and the workspace, or to `mine` and, if this
// is the first workgroup, the caller's arrays.
__device__ __forceinline__ void plan(const PageArgs& a, uint32_t (*sums)[kWaves], const Served* mine) {
  const bool tell = blockIdx.x == 0;
  const int64_t most = (int64_t)a.width << a.page_log2;
  const uint32_t n_free = clamped(a.counts[0], a.n_pages);
  uint32_t rows = 0, asked = 0, given = 0, refused = 0;
  for (int first = 0, turn = 0; first < a.n_seqs; first += kThreads, turn ^= 2) {
    const int i = first + (int)threadIdx.x;
    const bool there = i < a.n_seqs;
    const int len = there ? clamped(a.lens[i], most) : 0, more = there && a.change[i] > 0 ? a.change[i] : 0;
    uint32_t all;
    const uint32_t end = add(rows, block_sum(more, sums[turn], &all));
    rows = add(rows, all);
    bool served = len + (int64_t)more <= most && (more == 0 || end <= a.rows_cap);
    const uint32_t need = served ? (uint32_t)(pages_of(len + (int64_t)more, a.page_log2) - pages_of(len, a.page_log2)) : 0;
    const uint32_t upto = add(asked, block_sum(need, sums[turn + 1], &all));
    asked = add(asked, all);
    served = served && (need == 0 || upto <= n_free);
    given += served ? need : 0;
    refused += there && !served;
    if (there) {
      const int cu = end < INT32_MAX ? (int)end : INT32_MAX, start = served ? len : -1, now = served ? len + more : len;
      const int top = (int)(n_free - 1 - (upto - need));      // (unused by those that get none)
      if (tell) {
        a.cu[i + 1] = cu;
        a.start[i] = start;
        a.lens_out[i] = now;
      }
      if (mine) {
        mine->cu[i + 1] = cu;
        mine->start[i] = start;
        mine->len[i] = now;
        mine->top[i] = top;
      } else {
        a.ws[i] = top;
      }
    }
  }
  if (mine && threadIdx.x == 0) mine->cu[0] = 0;
  __syncthreads();
  if (!tell) return;
  uint32_t all;
  block_sum(given, sums[0], &all);
  const uint32_t left = n_free - all;
  block_sum(refused, sums[1], &all);
  if (threadIdx.x == 0) {
    a.cu[0] = 0;
    a.counts_out[0] = (int)left;
    a.counts_out[1] = (int)all;
  }
}

// Slot, position and the table's new entry of a row
__device__ __forceinline__ void fill_row(const PageArgs& a, const Served& s, int64_t row) {
  int64_t slot = -1;
  int pos = 0;
  if (row < s.cu[a.n_seqs]) {
    const int seq = rollout_of_pos(s.cu, 0, a.n_seqs, row), start = s.start[seq];
    const int at = (int)(row - s.cu[seq]);
    const int64_t to = (int64_t)(start < 0 ? s.len[seq] : start) + at;
    pos = to < INT32_MAX ? (int)to : INT32_MAX;              // (a refused sequence may ask for anything)
    if (start >= 0) {
      const int place = pos >> a.page_log2, fresh = (int)pages_of(start, a.page_log2);
      int page;
      if (place < fresh) {
        page = a.table[(int64_t)seq * a.width + place];
      } else {
        page = a.free_pages[s.top[seq] - (place - fresh)];
        if (at == 0 || (pos & ((1 << a.page_log2) - 1)) == 0) a.table[(int64_t)seq * a.width + place] = page;
      }
      if (page >= 0 && page < a.n_pages) slot = ((int64_t)page << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
    }
  }
  a.slots[row] = slot;
  if (a.pos) a.pos[row] = pos;
}

__global__ void __launch_bounds__(kThreads) reserve_plan_kernel(PageArgs a) {
  __shared__ uint32_t sums[4][kWaves];
  plan(a, sums, nullptr);
}

__global__ void __launch_bounds__(256) reserve_fill_kernel(PageArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row < a.rows_cap) fill_row(a, Served{a.cu, a.start, a.lens_out, a.ws}, row);
}

// Both in one launch for up to kThreads sequences: every workgroup plans for itself, which takes less than a launch (a batch of 192 sequences and 162 thousand rows 8.4 us and a
// second launch's host time in two, 5.6 in one; a step of 512 sequences 7.1 and 4.5).  Of many rows a workgroup takes one 1024 after another, so that each compute unit plans once: a million rows
// of 192 sequences 10.1 us, 4 million 27, room for as many of which a thousand are used 11.5 (with 512 workgroups 11.6, 27, 11.6; with one per 1024 rows 15, 52, 36; in two launches 13, 32, 13).
// With results in the place of inputs, which another workgroup may have yet to read, one workgroup takes all rows, up to kFewRows.
constexpr int kFewRows = 4096;
constexpr int64_t kPlans = 256;
__global__ void __launch_bounds__(kThreads) reserve_kernel(PageArgs a) {
  __shared__ uint32_t sums[4][kWaves];
  __shared__ int32_t cu[kThreads + 1], start[kThreads], len[kThreads], top[kThreads];
  const Served s{cu, start, len, top};
  plan(a, sums, &s);
  __syncthreads();
  for (int64_t row = (int64_t)blockIdx.x * kThreads + threadIdx.x; row < a.rows_cap; row += (int64_t)gridDim.x * kThreads) fill_row(a, s, row);
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
  __shared__ uint32_t sums[2][kWaves];
  uint32_t before = 0;
  for (int first = 0, turn = 0; first < a.n_seqs; first += kThreads, turn ^= 1) {
    const int i = first + (int)threadIdx.x;
    const uint32_t n = i < a.n_seqs ? a.ws[i] : 0;
    uint32_t all;
    const uint32_t to = add(before, block_sum(n, sums[turn], &all) - n);
    if (i < a.n_seqs) a.ws[i] = to < INT32_MAX ? (int)to : INT32_MAX;
    before = add(before, all);
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

struct Array { const void* at; int64_t bytes; };
bool same_memory(const Array& a, const Array& b) {
  const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
  return a.at && b.at && a.bytes > 0 && b.bytes > 0 && x < y + (uint64_t)b.bytes && y < x + (uint64_t)a.bytes;
}
// Whether an array that is written shares memory with another, which other workgroups may have yet to read or write.  The first two that are written, counts and lengths, may be the first two that
// are read.
template <int kWritten, int kRead>
bool overlap(const Array (&written)[kWritten], const Array (&read)[kRead]) {
  for (int i = 0; i < kWritten; ++i) {
    for (int j = i + 1; j < kWritten; ++j)
      if (same_memory(written[i], written[j])) return true;
    for (int j = 0; j < kRead; ++j)
      if (same_memory(written[i], read[j]) && !(i == j && i < 2 && written[i].at == read[j].at)) return true;
  }
  return false;
}

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
  const int64_t n4 = (int64_t)n_seqs * 4;
  if (overlap<8, 4>({{d_counts_out, 8}, {d_seq_lens_out, n4}, {d_block_table, n4 * table_width}, {d_start, n4}, {d_cu_new, n4 + 4}, {d_slots, rows_cap * 8},
                     {d_position_ids, rows_cap * 4}, {d_ws, n4}},
                    {{d_counts, 4}, {d_seq_lens, n4}, {d_new_lens, n4}, {d_free_pages, (int64_t)n_pages * 4}}))
    return NAT_INVALID_ARG;
  a.start = d_start;
  a.cu = d_cu_new;
  a.slots = d_slots;
  a.pos = d_position_ids;
  a.ws = (int32_t*)d_ws;
  a.rows_cap = rows_cap;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_PAGES, s);
  const bool in_place = d_counts_out == d_counts || d_seq_lens_out == d_seq_lens;
  if (n_seqs <= kThreads && (!in_place || rows_cap <= kFewRows)) {
    const int64_t blocks = in_place || rows_cap == 0 ? 1 : (rows_cap + kThreads - 1) / kThreads;
    reserve_kernel<<<(unsigned)(blocks < kPlans ? blocks : kPlans), kThreads, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
    return NAT_OK;
  }
  reserve_plan_kernel<<<1, kThreads, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  if (rows_cap == 0) return NAT_OK;
  reserve_fill_kernel<<<(unsigned)((rows_cap + 255) / 256), 256, 0, s>>>(a);
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
  const int64_t n4 = (int64_t)n_seqs * 4;
  if (overlap<4, 4>({{d_counts_out, 8}, {d_seq_lens_out, n4}, {d_free_pages, (int64_t)n_pages * 4}, {d_ws, n_seqs > 0 ? n4 + 4 : 0}},
                    {{d_counts, 4}, {d_seq_lens, n4}, {d_keep_lens, n4}, {d_block_table, n4 * table_width}}))
    return NAT_INVALID_ARG;
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
