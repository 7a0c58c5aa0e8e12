// Sampling the next token of every row from its logits: temperature, top-k, top-p, min-p, one given random word per row.
//
// Every logit has a whole-number weight a = round(2^40 2^y), y = (z - max) log2(e) / temperature in fp32.  Sums of whole numbers do not depend on their
// order, so which tokens are kept and which one is drawn is defined to the last bit, whatever order the wavefronts add in: an fp32 cumulative sum over a
// vocabulary leaves the draw to its rounding near every boundary.  2^40 keeps tokens down to 2^-41 of the likeliest one, and 2^20 weights fit 60 bits.
//
// One workgroup of 16 wavefronts per row.  It walks the row in slices of 1024 16-byte vectors, one per thread, so that a wavefront's part of a slice is 64
// vectors that follow one another: the draw, in order of index, goes by the sums of these parts, then by lanes, then by elements.
#include "nat_internal.h"

namespace nat {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxVocab = 1 << 20;
constexpr int kBins = 2048, kBinBits = 11;
constexpr uint32_t kKeyMinusInf = 0x007fffffu;        // order of -inf, below all that can be drawn
constexpr uint64_t kOne = 1ull << 40;

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int vocab;
  const uint32_t* random;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* ids;
  float *logp, *logq;
};

// whole numbers in the order of the logits; NaN as -inf, and zeros of both signs equal
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
  const uint32_t k = b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
  return z != z ? kKeyMinusInf : k;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __builtin_bit_cast(float, key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}

// (word * total) >> 32
__device__ __forceinline__ uint64_t share_of(uint32_t word, uint64_t total) {
  return word * (total >> 32) + ((word * (total & 0xffffffffu)) >> 32);
}

struct Weigher {
  uint32_t top;                  // key of the largest logit
  float max, per_nat;
  __device__ __forceinline__ uint64_t operator()(uint32_t key) const {
    if (key == top) return kOne;
    if (key <= kKeyMinusInf) return 0;
    const float y = (logit_of(key) - max) * per_nat;
    return y > -42.f ? (uint64_t)__double2ull_rn(exp2((double)y) * (double)kOne) : 0;
  }
};

// The row in vectors.  Vector j holds the elements j kE - lead .. + kE - 1; a vector that is wholly in the row is aligned.
template <class T>
struct Row {
  static constexpr int kE = 16 / sizeof(T);
  const T* p;
  int vocab, lead, vectors, slices;
  __device__ __forceinline__ Row(const void* logits, int64_t stride, int64_t row, int n) {
    p = (const T*)logits + row * stride;
    vocab = n;
    lead = (int)(((uintptr_t)p & 15) / sizeof(T));
    vectors = (n + lead + kE - 1) / kE;
    slices = (vectors + kThreads - 1) / kThreads;
  }
  __device__ __forceinline__ static uint32_t key(float z) { return key_of(z); }
  __device__ __forceinline__ static uint32_t key(uint16_t z) { return key_of(__builtin_bit_cast(float, (uint32_t)z << 16)); }
  // keys of vector j; outside the row: below all
  __device__ __forceinline__ void load(int j, uint32_t (&k)[kE]) const {
    const int e0 = j * kE - lead;
    if (e0 >= 0 && e0 + kE <= vocab) {
      union { uint4 q; T e[kE]; } x;
      x.q = *(const uint4*)(p + e0);
#pragma unroll
      for (int i = 0; i < kE; ++i) k[i] = key(x.e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kE; ++i) k[i] = e0 + i >= 0 && e0 + i < vocab ? key(p[e0 + i]) : 0;
    }
  }
};

struct Shared {
  uint64_t hist[kBins];
  uint64_t part[(kMaxVocab / 4 / kThreads + 2) * kWaves];     // sums of the wavefronts' parts of the slices
  uint64_t wave64[kWaves];
  double wave_f[kWaves];
  uint64_t found64;
  uint32_t found;
  int equal_end;
};

__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor((unsigned long long)x, d, 64);
  return x;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {       // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)x, d, 64);
    if (lane >= d) x += y;
  }
  return x;
}

// over the workgroup; every thread gets the result
__device__ __forceinline__ uint64_t block_sum64(uint64_t x, Shared& sm) {
  x = wave_sum64(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm.wave64[threadIdx.x >> 6] = x;
  __syncthreads();
  uint64_t s = 0;
  for (int w = 0; w < kWaves; ++w) s += sm.wave64[w];
  return s;
}

// The entry of x[0 .. n) in which the running sum passes `target`, i.e. the first whose inclusive sum is > target, and the sum before it; n if none is.
__device__ __forceinline__ int block_find(const uint64_t* x, int n, uint64_t target, uint64_t* before, Shared& sm) {
  const int per = (n + kThreads - 1) / kThreads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lo = threadIdx.x * per < n ? threadIdx.x * per : n, hi = lo + per < n ? lo + per : n;
  uint64_t mine = 0;
  for (int i = lo; i < hi; ++i) mine += x[i];
  const uint64_t incl = wave_scan64(mine);
  __syncthreads();
  if (lane == 63) sm.wave64[wave] = incl;
  if (threadIdx.x == 0) sm.found = (uint32_t)n;
  __syncthreads();
  uint64_t at = incl - mine;
  for (int w = 0; w < wave; ++w) at += sm.wave64[w];
  if (at <= target && target < at + mine) {
    for (int i = lo; i < hi; ++i) {
      if (target < at + x[i]) {
        sm.found = (uint32_t)i;
        sm.found64 = at;
        break;
      }
      at += x[i];
    }
  }
  __syncthreads();
  *before = sm.found64;
  return (int)sm.found;
}

// The largest key whose elements, with all above it, have a weight (an element's: of(key)) over `target` in all: narrowed down by histograms of the keys from
// `hi` down to `lo`.  *above: the weight above that key.  False if all of lo .. hi together do not pass the target.
template <class T, class Of>
__device__ __forceinline__ bool select_key(const Row<T>& row, uint32_t lo, uint32_t hi, uint64_t target, const Of& of, uint32_t* key, uint64_t* above, Shared& sm) {
  uint64_t over = 0;
  if (lo > hi) return false;
  for (;;) {
    const int bits = 32 - __clz(hi - lo), shift = hi == lo || bits <= kBinBits ? 0 : bits - kBinBits;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    for (int s = 0; s < row.slices; ++s) {
      const int j = s * kThreads + threadIdx.x;
      if (j >= row.vectors) break;
      uint32_t k[Row<T>::kE];
      row.load(j, k);
#pragma unroll
      for (int i = 0; i < Row<T>::kE; ++i)
        if (k[i] >= lo && k[i] <= hi) {
          const uint64_t a = of(k[i]);
          if (a) atomicAdd((unsigned long long*)&sm.hist[(hi - k[i]) >> shift], (unsigned long long)a);
        }
    }
    __syncthreads();
    uint64_t before;
    const int bin = block_find(sm.hist, kBins, target - over, &before, sm);
    if (bin == kBins) return false;
    over += before;
    hi -= (uint32_t)bin << shift;
    if (shift == 0) {
      *key = hi;
      *above = over;
      return true;
    }
    const uint32_t least = hi - ((1u << shift) - 1);
    if (least > lo && least <= hi) lo = least;
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  __shared__ Shared sm;
  constexpr int kE = Row<T>::kE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, a.row_stride, r, a.vocab);

  uint32_t top = 0;
  for (int s = 0; s < row.slices; ++s) {
    const int j = s * kThreads + threadIdx.x;
    if (j >= row.vectors) break;
    uint32_t k[kE];
    row.load(j, k);
#pragma unroll
    for (int i = 0; i < kE; ++i) top = k[i] > top ? k[i] : top;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d, 64);
    top = o > top ? o : top;
  }
  if (lane == 0) sm.wave64[wave] = top;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) top = sm.wave64[w] > top ? (uint32_t)sm.wave64[w] : top;
  if (top <= kKeyMinusInf) {                 // nothing to draw
    if (threadIdx.x == 0) {
      a.ids[r] = -1;
      if (a.logp) a.logp[r] = NAN;
      if (a.logq) a.logq[r] = NAN;
    }
    return;
  }
  const float temperature = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(temperature > 0.f);
  const Weigher weight{top, logit_of(top), 1.44269504088896341f / temperature};
  auto one = [](uint32_t) -> uint64_t { return 1; };

  // what stays: keys above `least`, and of those equal to it the first n_least
  uint32_t least = kKeyMinusInf;
  uint64_t n_least = 0;
  if (greedy) {
    least = top;
    n_least = 1;
  } else {
    const int32_t top_k = a.top_k ? a.top_k[r] : 0;
    if (top_k > 0 && top_k < a.vocab) {
      uint64_t above;
      if (select_key(row, kKeyMinusInf + 1, top, (uint64_t)top_k - 1, one, &least, &above, sm)) n_least = top_k - above;
    }
    const float top_p = a.top_p ? a.top_p[r] : 1.f;
    if (top_p < 1.f) {
      uint64_t total = 0;
      for (int s = 0; s < row.slices; ++s) {
        const int j = s * kThreads + threadIdx.x;
        if (j >= row.vectors) break;
        uint32_t k[kE];
        row.load(j, k);
#pragma unroll
        for (int i = 0; i < kE; ++i) total += k[i] > least ? weight(k[i]) : 0;
      }
      const uint64_t at_least = weight(least);
      total = block_sum64(total, sm) + n_least * at_least;
      const double share = top_p > 0.f ? (double)top_p * 4294967296.0 : 0.0;
      uint64_t reach = share_of((uint32_t)share, total);
      if (reach < 1) reach = 1;
      uint32_t key;
      uint64_t above;
      if (select_key(row, least + 1, top, reach - 1, weight, &key, &above, sm)) {
        least = key;
        const uint64_t each = weight(key);
        n_least = (reach - above + each - 1) / each;
      } else if (n_least > 0) {
        // the equal ones at the top-k's end: what is left after all above them
        uint64_t over = total - n_least * at_least;
        const uint64_t n = at_least ? (reach - over + at_least - 1) / at_least : 0;
        n_least = n < n_least ? n : n_least;
      }
    }
  }
  uint64_t weight_least = 1;
  if (!greedy && a.min_p) {
    const float min_p = a.min_p[r];
    if (min_p > 0.f) weight_least = (uint64_t)ceil((double)(min_p < 1.f ? min_p : 1.f) * (double)kOne);
  }

  // of the equal ones, the first n_least in order of index: up to index `equal_end`
  int equal_end = -1;
  if (n_least > 0) {
    for (int s = 0; s < row.slices; ++s) {
      const int j = s * kThreads + threadIdx.x;
      uint64_t n = 0;
      if (j < row.vectors) {
        uint32_t k[kE];
        row.load(j, k);
#pragma unroll
        for (int i = 0; i < kE; ++i) n += k[i] == least;
      }
      n = wave_sum64(n);
      if (lane == 0) sm.part[s * kWaves + wave] = n;
    }
    uint64_t before;
    __syncthreads();
    const int part = block_find(sm.part, row.slices * kWaves, n_least - 1, &before, sm);
    if (part == row.slices * kWaves) {
      equal_end = a.vocab;
    } else {
      const int j = part * 64 + lane;
      uint32_t k[kE];
      uint64_t n = 0;
      if (j < row.vectors) {
        row.load(j, k);
#pragma unroll
        for (int i = 0; i < kE; ++i) n += k[i] == least;
      }
      uint64_t at = before + wave_scan64(n) - n;
      if (n && at < n_least && n_least <= at + n) {
#pragma unroll
        for (int i = 0; i < kE; ++i)
          if (k[i] == least && ++at == n_least) sm.equal_end = j * kE - row.lead + i;
      }
      __syncthreads();
      equal_end = sm.equal_end;
    }
  }
  auto kept = [&](uint32_t key, int index) -> uint64_t {
    if (key < least || (key == least && index > equal_end)) return 0;
    const uint64_t w = greedy ? kOne : weight(key);
    return w >= weight_least ? w : 0;
  };

  // the draw, and the sum of the soft-max over the whole row
  double soft = 0.0;
  uint64_t total = 0;
  __syncthreads();
  for (int s = 0; s < row.slices; ++s) {
    const int j = s * kThreads + threadIdx.x;
    uint64_t w = 0;
    if (j < row.vectors) {
      uint32_t k[kE];
      row.load(j, k);
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        w += kept(k[i], j * kE - row.lead + i);
        if (a.logp && k[i] > kKeyMinusInf) soft += k[i] == top ? 1.f : __expf(logit_of(k[i]) - weight.max);
      }
    }
    total += w;
    w = wave_sum64(w);
    if (lane == 0) sm.part[s * kWaves + wave] = w;
  }
  total = block_sum64(total, sm);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) soft += __shfl_xor(soft, d, 64);
  if (lane == 0) sm.wave_f[wave] = soft;
  const uint64_t target = share_of(a.random[r], total);
  uint64_t before;
  const int part = block_find(sm.part, row.slices * kWaves, target, &before, sm);
  if (wave != 0) return;
  const int j = part * 64 + lane;
  uint32_t k[kE];
  uint64_t w[kE], sum = 0;
#pragma unroll
  for (int i = 0; i < kE; ++i) w[i] = 0;
  if (j < row.vectors) {
    row.load(j, k);
#pragma unroll
    for (int i = 0; i < kE; ++i) sum += w[i] = kept(k[i], j * kE - row.lead + i);
  }
  uint64_t at = before + wave_scan64(sum) - sum;
  if (sum && at <= target && target < at + sum) {
    bool done = false;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      if (!done && target < at + w[i]) {
        done = true;
        double all = 0.0;
        for (int x = 0; x < kWaves; ++x) all += sm.wave_f[x];
        a.ids[r] = j * kE - row.lead + i;
        if (a.logp) a.logp[r] = (float)((k[i] == top ? 0.0 : (double)(logit_of(k[i]) - weight.max)) - log(all));
        if (a.logq) a.logq[r] = (float)log((double)w[i] / (double)total);
      }
      at += w[i];
    }
  }
}

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" nat_status nat_sample(const void* d_logits, int64_t row_stride, int32_t n_rows, int32_t V, int32_t dtype, const uint32_t* d_random,
                                 const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int32_t* d_ids,
                                 float* d_logp, float* d_logq, void* stream) {
  if (dtype != NAT_DTYPE_F32 && dtype != NAT_DTYPE_BF16) return NAT_UNSUPPORTED_DTYPE;
  if (n_rows < 0) return NAT_INVALID_ARG;
  if (V <= 0 || V > kMaxVocab || (row_stride != 0 && row_stride < V)) return NAT_BAD_SHAPE;
  if (n_rows == 0) return NAT_OK;
  if (!d_logits || !d_random || !d_ids || ((uintptr_t)d_logits & (dtype == NAT_DTYPE_F32 ? 3 : 1))) return NAT_INVALID_ARG;
  SampleArgs a{d_logits, row_stride ? row_stride : V, V, d_random, d_temperature, d_top_p, d_min_p, d_top_k, d_ids, d_logp, d_logq};
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_SAMPLE, s);
  if (dtype == NAT_DTYPE_BF16) sample_kernel<uint16_t><<<n_rows, kThreads, 0, s>>>(a);
  else sample_kernel<float><<<n_rows, kThreads, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
