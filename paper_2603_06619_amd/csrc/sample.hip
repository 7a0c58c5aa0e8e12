// Sampling the next token of every row from its logits: temperature, top-k, top-p, min-p, one given random word per row.
//
// Every logit has a whole-number weight a = 2^40 2^y to the nearest, y = (z - max) log2(e) / temperature in fp32.  Sums of whole numbers do not depend on
// their order, so which tokens are kept and which one is drawn does not depend on how a row is dealt to wavefronts: an fp32 cumulative sum over a vocabulary
// leaves the draw to its rounding near every boundary.  2^40 keeps tokens down to 2^-41 of the likeliest one, and 2^20 weights fit 60 bits.
//
// A row is cut into ranges of 16-byte vectors, one per wavefront, 8 or more wavefronts per workgroup and 1 or more workgroups ("splits") per row.  Phase 1: the
// largest logit.  Phase 2: weights, and their sums over parts of the ranges; in rows with a top-k or top-p also a list of the tokens with at least 2^-12 of the
// largest weight, the candidates.  Phase 3, one workgroup per row: the draw, in order of index, by the sums of the parts, then by lanes, then by
// elements; in ranked rows first the least logit that stays, by histograms over the candidates, and the draw among them.  If what stays reaches
// below the candidates, or these are too many, the row is gone over again by phase 3 alone (draw_slowly).
#include "nat_internal.h"

namespace nat {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxSplits = 32;
constexpr int kUnroll = 4;                            // vectors per lane and step, and per part of a wavefront's range
constexpr int kBins = 1024, kBinBits = 10;
constexpr int kCandPerWave = 768;                     // capacity of a wavefront's list of candidates
constexpr int kCandRow = kCandPerWave * kWaves;       // of a row's, where two workgroups share a compute unit's LDS
constexpr int kCandSplit = 2 * kCandRow;              // where a row has several workgroups, and the last one the compute unit
constexpr float kCandReach = -12.f;                   // y of the last candidates
constexpr uint32_t kKeyMinusInf = 0x007fffffu;        // order of -inf, below all that can be drawn
constexpr uint64_t kOne = 1ull << 40;
constexpr float kLog2E = 1.44269504088896341f;

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int vocab, splits;
  const uint32_t* random;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* ids;
  float *logp, *logq;
  char* ws;
  size_t ws_row;                 // bytes per row
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
  float max, per_nat;            // of +inf: the largest finite value, as the logits that are +inf
  __device__ __forceinline__ Weigher(uint32_t top, float temperature) {
    max = fminf(logit_of(top), __FLT_MAX__);
    per_nat = fmaxf(fminf(kLog2E / temperature, __FLT_MAX__), __FLT_MIN__);      // 0 * per_nat is 0, inf * per_nat is inf
  }
  // the median of three: +inf is 0 like the largest finite logit, NaN the lesser bound, whose weight is 0
  __device__ __forceinline__ float exponent(float z) const { return __builtin_amdgcn_fmed3f((z - max) * per_nat, -60.f, 0.f); }
  // 2^y = 2^n 2^f, f in [-1/2, 1/2], by the polynomial that meets 2^f at the ten Chebyshev points of the interval: relative error below 2^-44.  Adding
  // 2^52 rounds 2^(40 + y) to a whole number, which then is the low bits of the sum; in all 23 instructions
  static __device__ __forceinline__ uint64_t weight(float y) {
    const float n = rintf(y);
    const double f = (double)(y - n);
    double p = 0x1.b6571d9fbc782p-24;
    p = fma(p, f, 0x1.63ef9699f65f0p-20);
    p = fma(p, f, 0x1.ffcb7678dfe12p-17);
    p = fma(p, f, 0x1.43088e257f900p-13);
    p = fma(p, f, 0x1.5d87fe908f6f7p-10);
    p = fma(p, f, 0x1.3b2ab72b175e9p-7);
    p = fma(p, f, 0x1.c6b08d704411ap-5);
    p = fma(p, f, 0x1.ebfbdff8149f2p-3);
    p = fma(p, f, 0x1.62e42fefa39f7p-1);
    p = fma(p, f, 1.0);
    const double scale = __builtin_bit_cast(double, (uint64_t)(uint32_t)((int)n + 1023 + 40) << 52);
    return __builtin_bit_cast(uint64_t, fma(p, scale, 0x1p52)) & ((1ull << 52) - 1);
  }
  __device__ __forceinline__ uint64_t of_key(uint32_t key) const { return key <= kKeyMinusInf ? 0 : weight(exponent(logit_of(key))); }
};

// What a row's settings ask for
struct Settings {
  float temperature, top_p;
  int top_k;
  uint64_t least;                // least weight that min_p lets stay
  bool greedy, ranked;
  __device__ __forceinline__ Settings(const SampleArgs& a, int64_t r) {
    temperature = a.temperature ? a.temperature[r] : 1.f;
    greedy = !(temperature > 0.f);
    top_k = a.top_k ? a.top_k[r] : 0;
    if (top_k >= a.vocab) top_k = 0;
    top_p = a.top_p ? a.top_p[r] : 1.f;
    ranked = !greedy && (top_k > 0 || top_p < 1.f);
    const float min_p = a.min_p ? a.min_p[r] : 0.f;
    least = min_p > 0.f ? (uint64_t)ceil((double)(min_p < 1.f ? min_p : 1.f) * (double)kOne) : 1;
  }
};

// The row in vectors.  Vector j holds the elements j kE - lead .. + kE - 1; a vector that is wholly in the row is aligned.  Elements outside the row are -inf.
template <class T>
struct Row {
  static constexpr int kE = 16 / sizeof(T);
  const T* p;
  int vocab, lead, vectors, steps, parts;        // steps of 64 kUnroll vectors of a wavefront, for `waves` of them: one part each
  __device__ __forceinline__ Row(const SampleArgs& a, int64_t row, int waves) {
    p = (const T*)a.logits + row * a.row_stride;
    vocab = a.vocab;
    lead = (int)(((uintptr_t)p & 15) / sizeof(T));
    vectors = (vocab + lead + kE - 1) / kE;
    steps = (vectors + 64 * kUnroll * waves - 1) / (64 * kUnroll * waves);
    parts = steps * waves;
  }
  __device__ __forceinline__ static float value(float z) { return z; }
  __device__ __forceinline__ static float value(uint16_t z) { return __builtin_bit_cast(float, (uint32_t)z << 16); }
  union Vector { uint4 q; T e[kE]; };
  __device__ __forceinline__ void load(int j, Vector& x) const {
    constexpr uint32_t kInf = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    const int e0 = j * kE - lead;
    x.q = make_uint4(kInf, kInf, kInf, kInf);
    if (e0 >= 0 && e0 + kE <= vocab) {
      x.q = *(const uint4*)(p + e0);
    } else if (j < vectors) {
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (e0 + i >= 0 && e0 + i < vocab) x.e[i] = p[e0 + i];
    }
  }
  __device__ __forceinline__ void load(int j, uint32_t (&k)[kE]) const {
    Vector x;
    load(j, x);
#pragma unroll
    for (int i = 0; i < kE; ++i) k[i] = key_of(value(x.e[i]));
  }
  // calls f(first vector of a part, vectors of this lane) for the parts of wavefront w
  template <class F>
  __device__ __forceinline__ void each_part(int w, const F& f) const {
    const int lane = threadIdx.x & 63;
    for (int s = 0; s < steps; ++s) {
      const int j0 = (w * steps + s) * (64 * kUnroll);
      Vector x[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) load(j0 + u * 64 + lane, x[u]);
      f(w * steps + s, j0, x);
    }
  }
};

struct Candidate { uint32_t key, index; };

// What phases 1 and 2 leave of a row: in LDS, or with more than one workgroup per row in the workspace
struct WaveSums { uint64_t all; double soft; };      // all weights; exponentials at temperature 1, where the weights are of another

constexpr int kMaxParts = kMaxVocab / 4 / (64 * kUnroll) + kMaxSplits * kWaves + 2;

template <int kCand>
struct SharedOf {
  static constexpr int kCandidates = kCand;
  uint64_t hist[kBins];
  uint64_t part[kMaxParts];
  union {
    Candidate cand[kCand];
    uint64_t slice[(kMaxVocab / 4 / kThreads + 2) * kWaves];     // draw_slowly: sums of the wavefronts' parts of the slices
  };
  WaveSums sums[kMaxSplits * kWaves];
  uint32_t top[kMaxSplits * kWaves];
  uint32_t cand_n[kMaxSplits * kWaves];
  uint64_t wave64[kWaves];
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
template <class Shared>
__device__ __forceinline__ uint64_t block_sum64(uint64_t x, Shared& sm) {
  x = wave_sum64(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm.wave64[threadIdx.x >> 6] = x;
  __syncthreads();
  uint64_t s = 0;
  for (int w = 0; w < kWaves; ++w) s += sm.wave64[w];
  return s;
}

// The i in [0, n) at which the running sum of x(i) passes `target`, i.e. the first whose inclusive sum is > target, and the sum before it; n if
// there is none.  What x reads has been written behind a barrier.
template <class X, class Shared>
__device__ __forceinline__ int block_find(const X& x, int n, uint64_t target, uint64_t* before, Shared& sm) {
  const int per = (n + kThreads - 1) / kThreads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lo = threadIdx.x * per < n ? threadIdx.x * per : n, hi = lo + per < n ? lo + per : n;
  uint64_t mine = 0;
  for (int i = lo; i < hi; ++i) mine += x(i);
  const uint64_t incl = wave_scan64(mine);
  __syncthreads();
  if (lane == 63) sm.wave64[wave] = incl;
  if (threadIdx.x == 0) sm.found = (uint32_t)n;
  __syncthreads();
  uint64_t at = incl - mine;
  for (int w = 0; w < wave; ++w) at += sm.wave64[w];
  if (at <= target && target < at + mine) {
    for (int i = lo; i < hi; ++i) {
      const uint64_t xi = x(i);
      if (target < at + xi) {
        sm.found = (uint32_t)i;
        sm.found64 = at;
        break;
      }
      at += xi;
    }
  }
  __syncthreads();
  *before = sm.found64;
  return (int)sm.found;
}

// The largest key whose elements, with all above it, have a weight (an element's: of(key)) over `target` in all: narrowed down by histograms of the keys from
// `hi` down to `lo`.  each(f) calls f(key) for every element.  *above: the weight above that key.  False if all of lo .. hi together do not pass the target.
template <class Each, class Of, class Shared>
__device__ __forceinline__ bool select_key(const Each& each, uint32_t lo, uint32_t hi, uint64_t target, const Of& of, uint32_t* key, uint64_t* above, Shared& sm) {
  uint64_t over = 0;
  if (lo > hi) return false;
  for (;;) {
    const int bits = 32 - __clz(hi - lo), shift = hi == lo || bits <= kBinBits ? 0 : bits - kBinBits;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    each([&](uint32_t k) {
      if (k >= lo && k <= hi) {
        const uint64_t a = of(k);
        if (a) atomicAdd((unsigned long long*)&sm.hist[(hi - k) >> shift], (unsigned long long)a);
      }
    });
    __syncthreads();
    uint64_t before;
    const int bin = block_find([&](int i) { return sm.hist[i]; }, kBins, target - over, &before, sm);
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

// What stays by rank: keys above `least`, and of those equal to it the first n_least.  each, of as in select_key; total_of(least): the weight above a key.
struct Ranked { uint32_t least; uint64_t n_least; };
template <class Each, class TotalOver, class Shared>
__device__ __forceinline__ Ranked rank_row(const Settings& set, const Weigher& weigh, uint32_t top, const Each& each, const TotalOver& total_over, Shared& sm) {
  Ranked r{kKeyMinusInf, 0};
  uint64_t above;
  if (set.top_k > 0 && select_key(each, kKeyMinusInf + 1, top, (uint64_t)set.top_k - 1, [](uint32_t) -> uint64_t { return 1; }, &r.least, &above, sm))
    r.n_least = set.top_k - above;
  if (!(set.top_p < 1.f)) return r;
  const uint64_t at_least = weigh.of_key(r.least), over = total_over(r.least), total = over + r.n_least * at_least;
  const double share = set.top_p > 0.f ? (double)set.top_p * 4294967296.0 : 0.0;
  uint64_t reach = share_of((uint32_t)share, total);
  if (reach < 1) reach = 1;
  uint32_t key;
  if (select_key(each, r.least + 1, top, reach - 1, [&](uint32_t k) { return weigh.of_key(k); }, &key, &above, sm)) {
    const uint64_t one = weigh.of_key(key);
    return Ranked{key, (reach - above + one - 1) / one};
  }
  // the equal ones at the top-k's end: what is left after all above them
  const uint64_t n = at_least ? (reach - over + at_least - 1) / at_least : 0;
  if (n < r.n_least) r.n_least = n;
  return r;
}

struct Drawn { int index; uint32_t key; uint64_t weight, total; };

__device__ __forceinline__ void write_out(const SampleArgs& a, int64_t r, const Drawn& d, const Weigher& weigh, double soft) {
  const float z = fminf(logit_of(d.key), __FLT_MAX__);
  a.ids[r] = d.index;
  if (a.logp) a.logp[r] = (float)((double)(z - weigh.max) - log(soft));
  if (a.logq) a.logq[r] = (float)log((double)d.weight / (double)d.total);
}

// A ranked row whose candidates do not do: everything from the row itself, in slices of one vector per thread.
template <class T, class Shared>
__device__ __noinline__ void draw_slowly(const SampleArgs& a, int64_t r, const Row<T>& row, const Settings& set, const Weigher& weigh, uint32_t top, double soft,
                                         Shared& sm) {
  constexpr int kE = Row<T>::kE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slices = (row.vectors + kThreads - 1) / kThreads;
  auto each = [&](auto f) {
    for (int s = 0; s < slices; ++s) {
      uint32_t k[kE];
      row.load(s * kThreads + threadIdx.x, k);
#pragma unroll
      for (int i = 0; i < kE; ++i) f(k[i]);
    }
  };
  const Ranked stay = rank_row(set, weigh, top, each, [&](uint32_t least) {
    uint64_t t = 0;
    each([&](uint32_t k) { t += k > least ? weigh.of_key(k) : 0; });
    return block_sum64(t, sm);
  }, sm);
  // of the equal ones, the first n_least in order of index: up to index `equal_end`
  auto in_slices = [&](auto f) {              // sums of f(key, index) over the wavefronts' parts of the slices
    __syncthreads();
    for (int s = 0; s < slices; ++s) {
      const int j = s * kThreads + threadIdx.x;
      uint32_t k[kE];
      row.load(j, k);
      uint64_t n = 0;
#pragma unroll
      for (int i = 0; i < kE; ++i) n += f(k[i], j * kE - row.lead + i);
      n = wave_sum64(n);
      if (lane == 0) sm.slice[s * kWaves + wave] = n;
    }
    __syncthreads();
  };
  auto slice = [&](int i) { return sm.slice[i]; };
  int equal_end = -1;
  if (stay.n_least > 0) {
    in_slices([&](uint32_t k, int) -> uint64_t { return k == stay.least; });
    uint64_t before;
    const int part = block_find(slice, slices * kWaves, stay.n_least - 1, &before, sm);
    equal_end = a.vocab;
    if (part < slices * kWaves) {
      const int j = part * 64 + lane;
      uint32_t k[kE];
      row.load(j, k);
      uint64_t n = 0;
#pragma unroll
      for (int i = 0; i < kE; ++i) n += k[i] == stay.least;
      uint64_t at = before + wave_scan64(n) - n;
      if (n && at < stay.n_least && stay.n_least <= at + n) {
#pragma unroll
        for (int i = 0; i < kE; ++i)
          if (k[i] == stay.least && ++at == stay.n_least) sm.equal_end = j * kE - row.lead + i;
      }
      __syncthreads();
      equal_end = sm.equal_end;
    }
  }
  auto kept = [&](uint32_t key, int index) -> uint64_t {
    if (key < stay.least || (key == stay.least && index > equal_end)) return 0;
    const uint64_t w = weigh.of_key(key);
    return w >= set.least ? w : 0;
  };
  in_slices(kept);
  uint64_t total = 0;
  for (int i = threadIdx.x; i < slices * kWaves; i += kThreads) total += sm.slice[i];
  total = block_sum64(total, sm);
  const uint64_t target = share_of(a.random[r], total);
  uint64_t before;
  const int part = block_find(slice, slices * kWaves, target, &before, sm);
  if (wave != 0) return;
  const int j = part * 64 + lane;
  uint32_t k[kE];
  row.load(j, k);
  uint64_t w[kE], sum = 0;
#pragma unroll
  for (int i = 0; i < kE; ++i) sum += w[i] = kept(k[i], j * kE - row.lead + i);
  uint64_t at = before + wave_scan64(sum) - sum;
  if (sum && at <= target && target < at + sum) {
    Drawn d{-1, 0, 0, total};
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      if (d.index < 0 && target < at + w[i]) d = Drawn{j * kE - row.lead + i, k[i], w[i], total};
      at += w[i];
    }
    write_out(a, r, d, weigh, soft);
  }
}

// Phase 1, wavefront w of the row's: its largest key
template <class T>
__device__ __forceinline__ uint32_t largest_key(const Row<T>& row, int w) {
  uint32_t top = 0;
  row.each_part(w, [&](int, int, const typename Row<T>::Vector (&x)[kUnroll]) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int i = 0; i < Row<T>::kE; ++i) {
        const uint32_t k = key_of(Row<T>::value(x[u].e[i]));
        top = k > top ? k : top;
      }
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d, 64);
    top = o > top ? o : top;
  }
  return top;
}

// Phase 2, wavefront w of the row's: sums of its parts to `part`, sums over all of them, candidates
template <class T>
__device__ __forceinline__ void weigh_range(const Row<T>& row, int w, const Settings& set, const Weigher& weigh, bool want_soft, uint64_t* part, WaveSums* sums,
                                            Candidate* cand, uint32_t* cand_n) {
  constexpr int kE = Row<T>::kE;
  using Vector = typename Row<T>::Vector;
  const int lane = threadIdx.x & 63;
  uint64_t all = 0;
  double soft = 0.0;
  if (set.greedy) {
    row.each_part(w, [&](int id, int, const Vector (&x)[kUnroll]) {
      uint64_t n = 0;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < kE; ++i) n += Row<T>::value(x[u].e[i]) >= weigh.max;
      n = wave_sum64(n);
      if (lane == 0) part[id] = n;
    });
  } else if (!set.ranked) {
    row.each_part(w, [&](int id, int, const Vector (&x)[kUnroll]) {
      uint64_t n = 0;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          const uint64_t a = Weigher::weight(weigh.exponent(Row<T>::value(x[u].e[i])));
          all += a;
          n += a >= set.least ? a : 0;
        }
      n = wave_sum64(n);
      if (lane == 0) part[id] = n;
    });
  } else {
    uint32_t n = 0;
    row.each_part(w, [&](int, int j0, const Vector (&x)[kUnroll]) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        uint32_t take = 0, at = n;
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          const float y = weigh.exponent(Row<T>::value(x[u].e[i]));
          all += Weigher::weight(y);
          const bool t = y >= kCandReach;
          take |= (uint32_t)t << i;
          const uint64_t b = __ballot(t);
          at = __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, at));
          n += __popcll(b);
        }
        if (take) {
          const int index = (j0 + u * 64 + lane) * kE - row.lead;
#pragma unroll
          for (int i = 0; i < kE; ++i)
            if (take >> i & 1) {
              if (at < kCandPerWave) cand[at] = Candidate{key_of(Row<T>::value(x[u].e[i])), (uint32_t)(index + i)};
              ++at;
            }
        }
      }
    });
    if (lane == 0) *cand_n = n;
  }
  if (want_soft && (set.greedy || set.temperature != 1.f)) {
    row.each_part(w, [&](int, int, const Vector (&x)[kUnroll]) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          const float e = __builtin_amdgcn_fmed3f((Row<T>::value(x[u].e[i]) - weigh.max) * kLog2E, -200.f, 0.f);       // NaN: 0
          soft += (double)__builtin_amdgcn_exp2f(e);
        }
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) soft += __shfl_xor(soft, d, 64);
  }
  all = wave_sum64(all);
  if (lane == 0) *sums = WaveSums{all, soft};
}

// Phase 3: what the `waves` wavefronts left is in sm (candidates in segments, `stride` of them for each wavefront)
template <class T, class Shared>
__device__ __forceinline__ void draw_row(const SampleArgs& a, int64_t r, const Row<T>& row, const Settings& set, const Weigher& weigh, uint32_t top, int waves,
                                         bool cand_overflow, int n_cand, Shared& sm) {
  constexpr int kE = Row<T>::kE;
  const int lane = threadIdx.x & 63;
  uint64_t all = 0;
  double soft = 0.0;
  for (int w = 0; w < waves; ++w) {
    all += sm.sums[w].all;
    soft += sm.sums[w].soft;
  }
  if (!set.greedy && set.temperature == 1.f) soft = (double)all * (1.0 / (double)kOne);
  if (set.ranked) {
    bool slow = cand_overflow;
    Ranked stay{};
    if (!slow) {
      auto each = [&](auto f) {
        for (int i = threadIdx.x; i < n_cand; i += kThreads) f(sm.cand[i].key);
      };
      // without a top-k the weight of the row, else of the candidates above the key
      bool all_of_row = true;
      if (set.top_k > n_cand) {
        slow = true;                           // the least of the top-k is no candidate
      } else {
        uint64_t cand_total = 0;
        each([&](uint32_t k) { cand_total += weigh.of_key(k); });
        cand_total = block_sum64(cand_total, sm);
        all_of_row = set.top_k <= 0;
        const double share = set.top_p > 0.f ? (double)set.top_p * 4294967296.0 : 0.0;
        if (all_of_row && share_of((uint32_t)share, all) > cand_total) {
          slow = true;                         // nor that of the top-p
        } else {
          stay = rank_row(set, weigh, top, each, [&](uint32_t least) {
            if (all_of_row) return all;
            uint64_t t = 0;
            each([&](uint32_t k) { t += k > least ? weigh.of_key(k) : 0; });
            return block_sum64(t, sm);
          }, sm);
        }
      }
    }
    if (slow) {
      draw_slowly(a, r, row, set, weigh, top, soft, sm);
      return;
    }
    // candidates are in order of index
    uint64_t before;
    int equal_end = -1;
    if (stay.n_least > 0) equal_end = block_find([&](int i) -> uint64_t { return sm.cand[i].key == stay.least; }, n_cand, stay.n_least - 1, &before, sm);
    auto kept = [&](int i) -> uint64_t {
      const uint32_t key = sm.cand[i].key;
      if (key < stay.least || (key == stay.least && i > equal_end)) return 0;
      const uint64_t w = weigh.of_key(key);
      return w >= set.least ? w : 0;
    };
    uint64_t total = 0;
    for (int i = threadIdx.x; i < n_cand; i += kThreads) total += kept(i);
    total = block_sum64(total, sm);
    const int i = block_find(kept, n_cand, share_of(a.random[r], total), &before, sm);
    if (threadIdx.x == 0) write_out(a, r, Drawn{(int)sm.cand[i].index, sm.cand[i].key, weigh.of_key(sm.cand[i].key), total}, weigh, soft);
    return;
  }
  uint64_t total = 0;
  for (int i = threadIdx.x; i < row.parts; i += kThreads) total += sm.part[i];
  total = block_sum64(total, sm);
  const uint64_t target = set.greedy ? 0 : share_of(a.random[r], total);
  uint64_t before;
  const int part = block_find([&](int i) { return sm.part[i]; }, row.parts, target, &before, sm);
  if (threadIdx.x >= 64) return;
  for (int u = 0; u < kUnroll; ++u) {
    const int j = (part * kUnroll + u) * 64 + lane;
    typename Row<T>::Vector x;
    row.load(j, x);
    uint64_t w[kE], sum = 0;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const float z = Row<T>::value(x.e[i]);
      w[i] = set.greedy ? (uint64_t)(z >= weigh.max) : Weigher::weight(weigh.exponent(z));
      if (w[i] < set.least && !set.greedy) w[i] = 0;
      sum += w[i];
    }
    const uint64_t incl = wave_scan64(sum);
    uint64_t at = before + incl - sum;
    const bool mine = sum && at <= target && target < at + sum;
    if (mine) {
      Drawn d{-1, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        if (d.index < 0 && target < at + w[i]) d = Drawn{j * kE - row.lead + i, key_of(Row<T>::value(x.e[i])), set.greedy ? 1 : w[i], set.greedy ? 1 : total};
        at += w[i];
      }
      write_out(a, r, d, weigh, soft);
    }
    if (__any(mine)) return;
    before += __shfl((unsigned long long)incl, 63, 64);
  }
}

__device__ __forceinline__ void nothing_to_draw(const SampleArgs& a, int64_t r) {
  a.ids[r] = -1;
  if (a.logp) a.logp[r] = NAN;
  if (a.logq) a.logq[r] = NAN;
}

// A workgroup per row: all three phases
template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_row_kernel(SampleArgs a) {
  __shared__ SharedOf<kCandRow> sm;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = blockIdx.x;
  const Row<T> row(a, r, kWaves);
  const uint32_t mine = largest_key(row, wave);
  if (lane == 0) sm.top[wave] = mine;
  __syncthreads();
  uint32_t top = 0;
  for (int w = 0; w < kWaves; ++w) top = sm.top[w] > top ? sm.top[w] : top;
  if (top <= kKeyMinusInf) {
    if (threadIdx.x == 0) nothing_to_draw(a, r);
    return;
  }
  const Settings set(a, r);
  const Weigher weigh(top, set.temperature);
  weigh_range(row, wave, set, weigh, a.logp != nullptr, sm.part, &sm.sums[wave], sm.cand + wave * kCandPerWave, &sm.cand_n[wave]);
  __syncthreads();
  int n_cand = 0;
  bool overflow = false;
  if (set.ranked) {                          // the segments close up
    Candidate c[kCandPerWave / 64];
    int to = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave) to = n_cand;
      overflow |= sm.cand_n[w] > kCandPerWave;
      n_cand += (int)sm.cand_n[w];
    }
    if (!overflow) {
      const int n = (int)sm.cand_n[wave];
#pragma unroll
      for (int i = 0; i < kCandPerWave / 64; ++i)
        if (64 * i + lane < n) c[i] = sm.cand[wave * kCandPerWave + 64 * i + lane];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kCandPerWave / 64; ++i)
        if (64 * i + lane < n) sm.cand[to + 64 * i + lane] = c[i];
      __syncthreads();
    }
  }
  draw_row(a, r, row, set, weigh, top, kWaves, overflow, n_cand, sm);
}

// Several workgroups per row: a kernel for each phase, what passes between them in the workspace
struct RowSpace {
  uint64_t* part;
  WaveSums* sums;
  uint32_t *top, *cand_n;
  Candidate* cand;               // kCandPerWave for each wavefront
};
__host__ __device__ inline size_t row_space(char* p, int parts, int waves, RowSpace* s) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = p ? p + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  s->part = (uint64_t*)take((size_t)parts * 8);
  s->sums = (WaveSums*)take((size_t)waves * sizeof(WaveSums));
  s->top = (uint32_t*)take((size_t)waves * 4);
  s->cand_n = (uint32_t*)take((size_t)waves * 4);
  s->cand = (Candidate*)take((size_t)waves * kCandPerWave * sizeof(Candidate));
  return at;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_top_kernel(SampleArgs a) {
  const int64_t r = blockIdx.x / a.splits;
  const int w = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % a.splits) * kWaves + (threadIdx.x >> 6)), waves = a.splits * kWaves;
  const Row<T> row(a, r, waves);
  RowSpace s;
  row_space(a.ws + r * a.ws_row, row.parts, waves, &s);
  const uint32_t top = largest_key(row, w);
  if ((threadIdx.x & 63) == 0) s.top[w] = top;
}

__device__ __forceinline__ uint32_t top_of_waves(const uint32_t* tops, int waves) {
  uint32_t top = 0;
  for (int i = threadIdx.x & 63; i < waves; i += 64) top = tops[i] > top ? tops[i] : top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d, 64);
    top = o > top ? o : top;
  }
  return top;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_weigh_kernel(SampleArgs a) {
  const int64_t r = blockIdx.x / a.splits;
  const int w = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % a.splits) * kWaves + (threadIdx.x >> 6)), waves = a.splits * kWaves;
  const Row<T> row(a, r, waves);
  RowSpace s;
  row_space(a.ws + r * a.ws_row, row.parts, waves, &s);
  const uint32_t top = top_of_waves(s.top, waves);
  if (top <= kKeyMinusInf) return;
  const Settings set(a, r);
  const Weigher weigh(top, set.temperature);
  weigh_range(row, w, set, weigh, a.logp != nullptr, s.part, &s.sums[w], s.cand + w * kCandPerWave, &s.cand_n[w]);
}

template <class T>
__global__ void __launch_bounds__(kThreads, 2) sample_draw_kernel(SampleArgs a) {
  __shared__ SharedOf<kCandSplit> sm;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = blockIdx.x;
  const int waves = a.splits * kWaves;
  const Row<T> row(a, r, waves);
  RowSpace s;
  row_space(a.ws + r * a.ws_row, row.parts, waves, &s);
  const uint32_t top = top_of_waves(s.top, waves);
  if (top <= kKeyMinusInf) {
    if (threadIdx.x == 0) nothing_to_draw(a, r);
    return;
  }
  const Settings set(a, r);
  const Weigher weigh(top, set.temperature);
  for (int i = threadIdx.x; i < waves; i += kThreads) {
    sm.sums[i] = s.sums[i];
    if (set.ranked) sm.cand_n[i] = s.cand_n[i];
  }
  if (!set.ranked)
    for (int i = threadIdx.x; i < row.parts; i += kThreads) sm.part[i] = s.part[i];
  __syncthreads();
  int n_cand = 0;
  bool overflow = false;
  if (set.ranked) {
    for (int w = 0; w < waves; ++w) {
      const int n = (int)sm.cand_n[w];
      if (n > kCandPerWave || n_cand + n > kCandSplit) {
        overflow = true;
        break;
      }
      if (w % kWaves == wave)
        for (int i = lane; i < n; i += 64) sm.cand[n_cand + i] = s.cand[w * kCandPerWave + i];
      n_cand += n;
    }
    __syncthreads();
  }
  draw_row(a, r, row, set, weigh, top, waves, overflow, n_cand, sm);
}

// Workgroups per row: enough for two on every compute unit
int splits_of(int64_t n_rows, int64_t V) {
  int64_t s = (512 + n_rows - 1) / n_rows;
  const int64_t most = (V + 4095) / 4096;              // at least 512 elements for a wavefront
  if (s > most) s = most;
  if (s > kMaxSplits) s = kMaxSplits;
  return (int)(s < 1 ? 1 : s);
}
// of a row that starts anywhere in its first vector
size_t row_bytes_of(int32_t V, int elem, int splits) {
  const int64_t e = 16 / elem, vectors = (V + (e - 1) + e - 1) / e, waves = splits * kWaves, per = 64 * kUnroll * waves;
  RowSpace s;
  return row_space(nullptr, (int)((vectors + per - 1) / per * waves), (int)waves, &s);
}

template <class T>
void launch(const SampleArgs& a, int32_t n_rows, hipStream_t s) {
  if (a.splits == 1) {
    sample_row_kernel<T><<<n_rows, kThreads, 0, s>>>(a);
    return;
  }
  sample_top_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
  sample_weigh_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
  sample_draw_kernel<T><<<n_rows, kThreads, 0, s>>>(a);
}

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" size_t nat_sample_workspace_bytes(int32_t n_rows, int32_t V, int32_t dtype) {
  if (n_rows <= 0 || V <= 0 || V > kMaxVocab || (dtype != NAT_DTYPE_F32 && dtype != NAT_DTYPE_BF16)) return 0;
  const int splits = splits_of(n_rows, V);
  return splits == 1 ? 0 : (size_t)n_rows * row_bytes_of(V, dtype == NAT_DTYPE_F32 ? 4 : 2, splits);
}

extern "C" nat_status nat_sample(const void* d_logits, int64_t row_stride, int32_t n_rows, int32_t V, int32_t dtype, const uint32_t* d_random,
                                 const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int32_t* d_ids,
                                 float* d_logp, float* d_logq, void* d_ws, size_t ws_bytes, void* stream) {
  if (dtype != NAT_DTYPE_F32 && dtype != NAT_DTYPE_BF16) return NAT_UNSUPPORTED_DTYPE;
  if (n_rows < 0) return NAT_INVALID_ARG;
  if (V <= 0 || V > kMaxVocab || (row_stride != 0 && row_stride < V)) return NAT_BAD_SHAPE;
  if (n_rows == 0) return NAT_OK;
  if (!d_logits || !d_random || !d_ids || ((uintptr_t)d_logits & (dtype == NAT_DTYPE_F32 ? 3 : 1))) return NAT_INVALID_ARG;
  const size_t need = nat_sample_workspace_bytes(n_rows, V, dtype);
  if (need > 0 && (!d_ws || ws_bytes < need)) return NAT_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)d_ws & 255) return NAT_INVALID_ARG;
  const int splits = splits_of(n_rows, V);
  SampleArgs a{d_logits, row_stride ? row_stride : V, V, splits, d_random, d_temperature, d_top_p, d_min_p, d_top_k, d_ids, d_logp, d_logq, (char*)d_ws,
               row_bytes_of(V, dtype == NAT_DTYPE_F32 ? 4 : 2, splits)};
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_SAMPLE, s);
  if (dtype == NAT_DTYPE_BF16) launch<uint16_t>(a, n_rows, s);
  else launch<float>(a, n_rows, s);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
