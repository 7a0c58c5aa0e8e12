// Sampling the next token of every row from its logits: temperature, top-k, top-p, min-p, one given random word per row.
//
// Every logit has a whole-number weight a = 2^40 2^y to the nearest, y = (z - max) log2(e) / temperature in fp32.  Sums of whole numbers do not depend on
// their order, so which tokens are kept and which one is drawn does not depend on how a row is dealt to wavefronts: an fp32 cumulative sum over a vocabulary
// leaves the draw to its rounding near every boundary.  2^40 keeps tokens down to 2^-41 of the likeliest one, and 2^20 weights fit 60 bits.
//
// A row is cut into parts of 128 16-byte vectors, dealt to wavefronts in turn, 8 wavefronts per workgroup and 1 or more workgroups ("splits") per row.
//   top      the largest logit;
//   bins     (rows with a top-k or top-p) a histogram of the exponents y, 1/16 apart: of tokens if the row has a top-k, else of their weight.  The bin in which
//            the top-k ends, or the weight that the top-p asks for;
//   list     the tokens of that bin (with a top-k and a top-p: of all bins down to it).  Among them the least logit that stays, and the last index that does of those
//            equal to it;
//   sums     weights of what stays, summed part by part;
//   draw     in order of index: by the sums of the parts, then by steps, lanes and elements.
// A row with one workgroup goes through them in one kernel; with more, each of top, bins, list and sums is a kernel, and the workgroup that comes last in
// a row does what follows from all (it knows by a counter; nobody waits).  If the list is longer than LDS has room for (very many equal logits), the row
// is gone over several times more by one workgroup (threshold_slowly).
//
// 512 rows of 152064 fp32 logits, no filter: 103 to 109 us for 311 MB, read twice (5.7 TB/s).  The 512 workgroups are all resident and in step: first all read for the
// maximum (50 us, vector pipes idle), then all compute weights (60 us of vector instructions, the memory idle), and the two add up.  Four rows of 151936 bf16 logits
// with every filter: 33 us, all of it latency (top 3.3, bins 7.8, list 8.4, sums 11.5, and three gaps between launches of 2): each phase reads a megabyte in 2 to 3 us, and
// its last workgroup then takes 3 to 5 for fences, loads of what the others wrote, and a search.
#include "nat_internal.h"

namespace nat {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxSplits = 32;
constexpr int kUnroll = 2;                            // vectors per lane and step, and per part
constexpr int kBins = 1024, kBinBits = 10;
constexpr float kBinsPerOctave = 16.f;                // of exponents: the last bin holds weights of 0 alone
constexpr int kList = 4096;                           // tokens of a list: two workgroups share a compute unit's LDS
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

// 2^40 2^(j / 64), j = 0 .. 63, in LDS
struct Powers {
  double of[64];
  __device__ __forceinline__ void fill() {           // read behind a barrier
    if (threadIdx.x < 64) of[threadIdx.x] = exp2((double)threadIdx.x * (1.0 / 64)) * (double)kOne;
  }
};

struct Weigher {
  const Powers* powers;
  float max, per_nat;            // of +inf: the largest finite value, as the logits that are +inf
  __device__ __forceinline__ Weigher(uint32_t top, float temperature, const Powers& p) : powers(&p) {
    max = fminf(logit_of(top), __FLT_MAX__);
    per_nat = fmaxf(fminf(kLog2E / temperature, __FLT_MAX__), __FLT_MIN__);      // 0 * per_nat is 0, inf * per_nat is inf
  }
  // the median of three: +inf is 0 like the largest finite logit, NaN the lesser bound, whose weight is 0
  __device__ __forceinline__ float exponent(float z) const { return __builtin_amdgcn_fmed3f((z - max) * per_nat, -60.f, 0.f); }
  // 2^y = 2^n 2^(j / 64) 2^r, |r| <= 1/128; 2^r - 1 = r (c1 + r (c2 + r (c3 + r c4))) through the four Chebyshev points of (2^r - 1) / r, all but the last two
  // steps in fp32: error below 2^-40 of the weight.  Adding 2^52 rounds to a whole number, which then is the low 52 bits (kBias: those above).  In all 24
  // instructions, six of them fp64; a polynomial of degree 9 without a table takes 38
  static constexpr uint64_t kBias = 0x433ull << 52;
  __device__ __forceinline__ uint64_t biased_weight(float y) const {
    constexpr float kWhole = 0x1.8p23f;              // adding it rounds to a whole number, the low bits of the sum
    const float t = fmaf(y, 64.f, kWhole), r = fmaf(t - kWhole, -1.f / 64, y);
    const uint32_t bits = __builtin_bit_cast(uint32_t, t);
    const uint64_t power = __builtin_bit_cast(uint64_t, powers->of[bits & 63]) + ((uint64_t)((bits & ~63u) << 14) << 32);
    const double p = __builtin_bit_cast(double, power);
    const float h = fmaf(fmaf(0x1.3b2acbp-7f, r, 0x1.c6b0b9p-5f), r, 0x1.ebfbe0p-3f);
    const double q = (double)r * fma((double)h, (double)r, 0x1.62e42fefa2417p-1);
    return __builtin_bit_cast(uint64_t, fma(p, 1.0 + q, 0x1p52));
  }
  __device__ __forceinline__ uint64_t weight(float y) const { return biased_weight(y) & ((1ull << 52) - 1); }
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
  int vocab, lead, vectors, waves, steps, parts;       // steps of 64 kUnroll vectors of every wavefront, one part each: side by side, so that a workgroup reads on
  __device__ __forceinline__ Row(const SampleArgs& a, int64_t row, int n_waves) {
    waves = n_waves;
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
  // The parts of wavefront w: f(first vector, this lane's vector) for every 64 vectors of a part, then end(part).  A part's vectors are loaded together, a part
  // ahead, and used in a loop that stays a loop: unrolled, code that runs a few times spends longer being fetched than running.  kBack: the last part
  // first.  Passes over a row go to and fro, so that each begins with what the one before it left in the caches (512 rows of 608 KB, 1.2 times
  // the Infinity Cache: 103 us, all passes forward 107)
  template <bool kBack, class F, class End>
  __device__ __forceinline__ void each_part(int w, const F& f, const End& end) const {
    const int lane = threadIdx.x & 63;
    Vector x[kUnroll], next[kUnroll];
    auto load_part = [&](int j0, Vector (&y)[kUnroll]) {
      if (j0 * kE - lead >= 0 && (j0 + 64 * kUnroll) * kE - lead <= vocab) {       // the same for all lanes
        const uint4* from = (const uint4*)(p + (j0 * kE - lead)) + lane;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) y[u].q = from[64 * u];
      } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) load(j0 + u * 64 + lane, y[u]);
      }
    };
    auto first = [&](int s) { return ((kBack ? steps - 1 - s : s) * waves + w) * (64 * kUnroll); };
    load_part(first(0), next);
    for (int s = 0; s < steps; ++s) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u].q = next[u].q;
      if (s + 1 < steps) load_part(first(s + 1), next);
#pragma unroll 1
      for (int u = 0; u < kUnroll; ++u) {
        f(first(s) + u * 64, x[0]);
#pragma unroll
        for (int v = 0; v + 1 < kUnroll; ++v) x[v].q = x[v + 1].q;
      }
      end(first(s) / (64 * kUnroll));
    }
  }
  template <bool kBack, class F>
  __device__ __forceinline__ void each_vector(int w, const F& f) const {
    each_part<kBack>(w, f, [](int) {});
  }
};

// What other workgroups read is written past the L2 of this XCD: a fence then finds nothing there to write back (1 us, else 4)
template <bool kOthers>
__device__ __forceinline__ void put(uint64_t* p, uint64_t x) {
  if constexpr (kOthers) __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *p = x;
}

typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
struct Listed { uint32_t key, index; };
struct WaveSums { uint64_t all; double soft; };      // all weights; exponentials at temperature 1, where the weights are of another
// The tokens that stay: keys above `least`, and those equal to it up to index `equal_end`
struct Stay {
  uint32_t least;
  int equal_end;
  __device__ __forceinline__ bool has(uint32_t key, int index) const { return key > least || (key == least && index <= equal_end); }
};
// What is listed: exponents' bins first .. last; what lies above them, tokens if the row has a top-k, else weight; the weight of the row (rows without a top-k)
struct Gather { int first, last; uint64_t above, all; };

constexpr int kMaxParts = kMaxVocab / 4 / (64 * kUnroll) + kMaxSplits * kWaves + 2;

struct Shared {
  Powers powers;
  __attribute__((aligned(16))) uint64_t hist[kBins];
  uint64_t part[kMaxParts];
  union {
    Listed list[kList];
    uint64_t slice[(kMaxVocab / 4 / kThreads + 2) * kWaves];     // threshold_slowly: sums of the wavefronts' parts of the slices
  };
  WaveSums sums[kMaxSplits * kWaves];
  uint32_t top[kWaves];
  uint64_t wave64[kWaves];
  uint64_t found64;
  uint32_t found, list_n;
  int equal_end, last_one;
};

// A value from another lane by way of the vector pipeline, 0 where the control has none: the sums below take a tenth of the time of their shuffles through LDS
template <int kControl, int kRows>
__device__ __forceinline__ uint64_t from_lane(uint64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, kControl, kRows, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), kControl, kRows, 0xf, false);
  return (uint64_t)hi << 32 | lo;
}
// inclusive: within rows of 16 lanes by 1, 2, 4, 8, then the last lane of rows 0 and 2 to rows 1 and 3, then lane 31 to rows 2 and 3
__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {
  x += from_lane<0x111, 0xf>(x);
  x += from_lane<0x112, 0xf>(x);
  x += from_lane<0x114, 0xf>(x);
  x += from_lane<0x118, 0xf>(x);
  x += from_lane<0x142, 0xa>(x);
  x += from_lane<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
  x = wave_scan64(x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, 63), hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), 63);
  return (uint64_t)hi << 32 | lo;
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

// The i in [0, n) at which the running sum of x(i) passes target(sum of all), i.e. the first whose inclusive sum is greater, the sum before it, and that of all;
// n if there is none.  What x reads has been written behind a barrier.
template <class X, class Target>
__device__ __forceinline__ int block_find(const X& x, int n, const Target& target_of, uint64_t* before, uint64_t* total, Shared& sm) {
  const int per = (n + kThreads - 1) / kThreads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lo = threadIdx.x * per < n ? threadIdx.x * per : n, hi = lo + per < n ? lo + per : n;
  uint64_t mine = 0;
  for (int i = lo; i < hi; ++i) mine += x(i);
  const uint64_t incl = wave_scan64(mine);
  __syncthreads();
  if (lane == 63) sm.wave64[wave] = incl;
  if (threadIdx.x == 0) sm.found = (uint32_t)n;
  __syncthreads();
  uint64_t at = incl - mine, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const uint64_t sum = sm.wave64[w];
    at += w < wave ? sum : 0;
    all += sum;
  }
  const uint64_t target = target_of(all);
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
  *total = all;
  return (int)sm.found;
}
template <class X>
__device__ __forceinline__ int block_find(const X& x, int n, uint64_t target, uint64_t* before, Shared& sm) {
  uint64_t total;
  return block_find(x, n, [&](uint64_t) { return target; }, before, &total, sm);
}

// The largest key whose elements, with all above it, have a weight (an element's: of(key)) over `target` in all: narrowed down by histograms of the keys from
// `hi` down to `lo`.  each(f) calls f(key) for every element.  *above: the weight above that key.  False if all of lo .. hi together do not pass the target.
template <class Each, class Of>
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

struct Drawn { int index; uint32_t key; uint64_t weight, total; };

__device__ __forceinline__ void write_out(const SampleArgs& a, int64_t r, const Drawn& d, const Weigher& weigh, double log_soft) {
  const float z = fminf(logit_of(d.key), __FLT_MAX__);
  a.ids[r] = d.index;
  if (a.logp) a.logp[r] = (float)((double)(z - weigh.max) - log_soft);
  if (a.logq) a.logq[r] = (float)log((double)d.weight / (double)d.total);
}
__device__ __forceinline__ void nothing_to_draw(const SampleArgs& a, int64_t r) {
  a.ids[r] = -1;
  if (a.logp) a.logp[r] = NAN;
  if (a.logq) a.logq[r] = NAN;
}

// weight that the top-p asks for, of a total
__device__ __forceinline__ uint64_t reach_of(float top_p, uint64_t total) {
  const double share = top_p > 0.f ? (double)top_p * 4294967296.0 : 0.0;
  const uint64_t reach = share_of((uint32_t)share, total);
  return reach < 1 ? 1 : reach;
}

// Keys above `least` and the first n_least of those equal to it stay by rank, of elements that each(f) calls f(key) for.  over_top: the weight above all of
// them, over(least): of them above a key; by_count: they hold the end of the top-k, over_top is the number of tokens above them, 0 if there is a top-p too.
struct Ranked { uint32_t least; uint64_t n_least; };
template <class Each, class Over>
__device__ __forceinline__ Ranked rank_tokens(const Settings& set, const Weigher& weigh, bool by_count, uint32_t lo, uint32_t hi, uint64_t total, uint64_t over_top,
                                              const Each& each, const Over& over, Shared& sm) {
  auto by_weight = [&](uint32_t k) { return weigh.of_key(k); };
  Ranked r{lo - 1, 0};
  uint64_t above, at_least = 0;
  if (by_count) {
    if (select_key(each, lo, hi, (uint64_t)set.top_k - over_top - 1, [](uint32_t) -> uint64_t { return 1; }, &r.least, &above, sm))
      r.n_least = set.top_k - over_top - above;
    if (!(set.top_p < 1.f)) return r;
    at_least = weigh.of_key(r.least);
    total = over(r.least) + r.n_least * at_least;
  }
  const uint64_t reach = reach_of(set.top_p, total);
  uint32_t key;
  if (select_key(each, r.least + 1, hi, reach - 1 - over_top, by_weight, &key, &above, sm)) {
    const uint64_t one = weigh.of_key(key);
    return Ranked{key, (reach - over_top - above + one - 1) / one};
  }
  // the equal ones at the top-k's end: what is left after all above them
  const uint64_t n = at_least ? (reach - (total - r.n_least * at_least) + at_least - 1) / at_least : 0;
  if (n < r.n_least) r.n_least = n;
  return r;
}

// A list that is too long: the least logit that stays from the row itself, in slices of one vector per thread.  512 fp32 rows of 152064 take 220 to 250 us with a
// top-p of 0.9, and this way 720 to 830 (temperature 5, 30), 840 (a top-k of 5000 as well), 1750 (all logits equal); 4 bf16 rows 35, and 260 to 290.  Its arguments come by value: had it references,
// the callers would keep theirs in memory from the start (5 us of the list kernel's 15).
template <class T>
__device__ __noinline__ Stay threshold_slowly(const Row<T> row, const Settings set, const Weigher weigh, uint32_t top, Shared& sm) {
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
  auto over = [&](uint32_t least) {
    uint64_t t = 0;
    each([&](uint32_t k) { t += k > least ? weigh.of_key(k) : 0; });
    return block_sum64(t, sm);
  };
  const Ranked r = rank_tokens(set, weigh, set.top_k > 0, kKeyMinusInf + 1, top, set.top_k > 0 ? 0 : over(kKeyMinusInf), 0, each, over, sm);
  if (r.n_least == 0) return Stay{r.least, -1};
  __syncthreads();
  for (int s = 0; s < slices; ++s) {
    uint32_t k[kE];
    row.load(s * kThreads + threadIdx.x, k);
    uint64_t n = 0;
#pragma unroll
    for (int i = 0; i < kE; ++i) n += k[i] == r.least;
    n = wave_sum64(n);
    if (lane == 0) sm.slice[s * kWaves + wave] = n;
  }
  __syncthreads();
  uint64_t before;
  const int part = block_find([&](int i) { return sm.slice[i]; }, slices * kWaves, r.n_least - 1, &before, sm);
  if (part == slices * kWaves) return Stay{r.least, row.vocab};
  const int j = part * 64 + lane;
  uint32_t k[kE];
  row.load(j, k);
  uint64_t n = 0;
#pragma unroll
  for (int i = 0; i < kE; ++i) n += k[i] == r.least;
  uint64_t at = before + wave_scan64(n) - n;
  if (n && at < r.n_least && r.n_least <= at + n) {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (k[i] == r.least && ++at == r.n_least) sm.equal_end = j * kE - row.lead + i;
  }
  __syncthreads();
  return Stay{r.least, sm.equal_end};
}

// top: the largest key of wavefront w's parts
template <class T>
__device__ __forceinline__ uint32_t largest_key(const Row<T>& row, int w) {
  float m = -INFINITY;                       // fmaxf passes NaN over
  row.template each_vector<false>(w, [&](int, const typename Row<T>::Vector& x) {
#pragma unroll
    for (int i = 0; i < Row<T>::kE; ++i) m = fmaxf(m, Row<T>::value(x.e[i]));
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  return key_of(m);
}

__device__ __forceinline__ int bin_of(float y) {
  const int b = (int)(y * -kBinsPerOctave);
  return b < kBins ? b : kBins - 1;
}

// bins: tokens or weights of the wavefront's parts, added to the histogram in LDS
template <class T>
__device__ __forceinline__ void bin_parts(const Row<T>& row, int w, const Settings& set, const Weigher& weigh, uint64_t* hist) {
  row.template each_vector<true>(w, [&](int, const typename Row<T>::Vector& x) {
#pragma unroll
    for (int i = 0; i < Row<T>::kE; ++i) {
      const float y = weigh.exponent(Row<T>::value(x.e[i]));
      if (y <= -60.f) continue;                // weight 0
      if (set.top_k > 0) atomicAdd((uint32_t*)&hist[bin_of(y)], 1u);
      else atomicAdd((unsigned long long*)&hist[bin_of(y)], (unsigned long long)weigh.weight(y));
    }
  });
}

// Which bins to list, from the row's histogram (all threads; behind a barrier)
__device__ __forceinline__ Gather choose_bins(const Settings& set, const uint64_t* hist, Shared& sm) {
  uint64_t above, all;
  const int bin = block_find([&](int i) { return hist[i]; }, kBins,
                             [&](uint64_t total) { return (set.top_k > 0 ? (uint64_t)set.top_k : reach_of(set.top_p, total)) - 1; }, &above, &all, sm);
  if (bin == kBins) return Gather{0, kBins - 1, 0, all};       // fewer tokens than the top-k: all of them
  return set.top_k > 0 && set.top_p < 1.f ? Gather{0, bin, 0, all} : Gather{bin, bin, above, all};
}

// list: the tokens in those bins, of the wavefront's parts; *n counts on past the room
template <class T>
__device__ __forceinline__ void list_parts(const Row<T>& row, int w, const Weigher& weigh, const Gather& g, Listed* list, uint32_t* n) {
  constexpr int kE = Row<T>::kE;
  const int lane = threadIdx.x & 63;
  row.template each_vector<false>(w, [&](int j, const typename Row<T>::Vector& x) {
    uint32_t take = 0;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const float y = weigh.exponent(Row<T>::value(x.e[i]));
      const int b = bin_of(y);
      take |= (uint32_t)(b >= g.first && b <= g.last && y > -60.f) << i;
    }
    if (take) {
      uint32_t at = atomicAdd(n, (uint32_t)__popc(take));
      const int index = (j + lane) * kE - row.lead;
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (take >> i & 1) {
          if (at < kList) list[at] = Listed{key_of(Row<T>::value(x.e[i])), (uint32_t)(index + i)};
          ++at;
        }
    }
  });
}

// What stays, from a list of up to kThreads tokens in LDS (in no order): one token per thread, which counts those in front of it (larger, or equal with a
// lower index).  Sorted, the last one that stays has the least logit and the last index among those equal to it.
__device__ __forceinline__ Stay threshold_of_short_list(const Settings& set, const Weigher& weigh, const Gather& g, int n, Shared& sm) {
  const int t = threadIdx.x;
  uint64_t* order = sm.hist;                   // tokens as whole numbers in that order; then their weights, sorted
  static_assert(kThreads + 2 <= kBins, "");
  const Listed mine = t < n ? sm.list[t] : Listed{0, 0};
  const uint64_t place = (uint64_t)mine.key << 32 | (uint32_t)~mine.index;
  __syncthreads();                             // the histogram is done with
  if (t < n) order[t] = place;
  if (t < 2) order[n + t] = 0;
  __syncthreads();
  int rank = 0;
  if ((t & ~63) < n) {
    for (int i = 0; i < n; i += 2) {
      const u64x2 x = *(const u64x2*)(order + i);
      rank += (x[0] > place) + (x[1] > place);
    }
  }
  __syncthreads();
  if (t < n) {
    order[rank] = weigh.of_key(mine.key);
    sm.list[rank] = mine;
  }
  __syncthreads();
  int end = n;                                 // tokens that stay
  if (set.top_k > 0 && set.top_k - (int)g.above < n) end = set.top_k - (int)g.above;
  if (set.top_k <= 0 || set.top_p < 1.f) {
    uint64_t before, total;
    const int last = block_find([&](int i) { return order[i]; }, end,
                                [&](uint64_t of_top_k) { return set.top_k > 0 ? reach_of(set.top_p, of_top_k) - 1 : reach_of(set.top_p, g.all) - 1 - g.above; }, &before, &total, sm);
    end = last < end ? last + 1 : end;
  }
  return Stay{sm.list[end - 1].key, (int)sm.list[end - 1].index};
}

// What stays, from the list in LDS (in no order)
__device__ __forceinline__ Stay threshold_of_list(const Settings& set, const Weigher& weigh, uint32_t top, const Gather& g, int n, Shared& sm) {
  if (n <= kThreads) return threshold_of_short_list(set, weigh, g, n, sm);
  auto each = [&](auto f) {
    for (int i = threadIdx.x; i < n; i += kThreads) f(sm.list[i].key);
  };
  uint32_t lo = top, hi = 0;
  each([&](uint32_t k) {
    lo = k < lo ? k : lo;
    hi = k > hi ? k : hi;
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_xor(lo, d, 64), y = __shfl_xor(hi, d, 64);
    lo = x < lo ? x : lo;
    hi = y > hi ? y : hi;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm.wave64[threadIdx.x >> 6] = (uint64_t)hi << 32 | lo;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    const uint32_t x = (uint32_t)sm.wave64[w], y = (uint32_t)(sm.wave64[w] >> 32);
    lo = x < lo ? x : lo;
    hi = y > hi ? y : hi;
  }
  const Ranked r = rank_tokens(set, weigh, set.top_k > 0, lo, hi, g.all, g.above, each, [&](uint32_t least) {
    uint64_t t = 0;
    each([&](uint32_t k) { t += k > least ? weigh.of_key(k) : 0; });
    return block_sum64(t, sm);
  }, sm);
  if (r.n_least == 0) return Stay{r.least, -1};
  // the n_least-th index of those equal to the least: in the order of ~index the largest come first
  uint32_t key;
  uint64_t above;
  const bool some = select_key([&](auto f) {
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (sm.list[i].key == r.least) f(~sm.list[i].index);
  }, ~(uint32_t)kMaxVocab, 0xffffffffu, r.n_least - 1, [](uint32_t) -> uint64_t { return 1; }, &key, &above, sm);
  return Stay{r.least, some ? (int)~key : kMaxVocab};
}

// sums: weights of what stays, of each of the wavefront's parts; of all their tokens, and (kSoft) their exponentials at temperature 1
template <bool kOthers, bool kSoft, class T>
__device__ __forceinline__ void sum_parts(const Row<T>& row, int w, const Settings& set, const Weigher& weigh, const Stay& stay, bool want_all, uint64_t* part,
                                          WaveSums* sums) {
  constexpr int kE = Row<T>::kE;
  using Vector = typename Row<T>::Vector;
  const int lane = threadIdx.x & 63;
  uint64_t all = 0, n = 0;
  double soft = 0.0;
  // In fp32, summed in fp64: the exponent's rounding is an error of 2^-24 |exponent| of a term, of either sign, so log-probs have one of 3e-8 to 5e-8 (in the weights' 40
  // bits, as at temperature 1, 2e-8, which is their own rounding; the weights would be computed twice)
  auto add_soft = [&](const Vector& x) {
    if constexpr (kSoft) {
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const float e = __builtin_amdgcn_fmed3f((Row<T>::value(x.e[i]) - weigh.max) * kLog2E, -200.f, 0.f);       // NaN: 0
        soft += (double)__builtin_amdgcn_exp2f(e);
      }
    }
  };
  auto end = [&](int id) {
    n = wave_sum64(n);
    if (lane == 0) put<kOthers>(part + id, n);
    n = 0;
  };
  if (set.greedy) {
    row.template each_part<true>(w, [&](int, const Vector& x) {
#pragma unroll
      for (int i = 0; i < kE; ++i) n += Row<T>::value(x.e[i]) >= weigh.max;
      add_soft(x);
    }, end);
  } else if (!set.ranked && set.least <= 1) {
    row.template each_part<true>(w, [&](int, const Vector& x) {
#pragma unroll
      for (int i = 0; i < kE; ++i) n += weigh.biased_weight(weigh.exponent(Row<T>::value(x.e[i])));
      add_soft(x);
    }, [&](int id) {
      n -= (uint64_t)(kE * kUnroll) * Weigher::kBias;
      all += n;
      end(id);
    });
  } else if (!set.ranked) {
    row.template each_part<true>(w, [&](int, const Vector& x) {
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const uint64_t a = weigh.weight(weigh.exponent(Row<T>::value(x.e[i])));
        all += a;
        n += a >= set.least ? a : 0;
      }
      add_soft(x);
    }, end);
  } else {
    row.template each_part<true>(w, [&](int j, const Vector& x) {
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const float z = Row<T>::value(x.e[i]);
        const bool stays = stay.has(key_of(z), (j + lane) * kE - row.lead + i);
        if (want_all || __any(stays)) {
          const uint64_t a = weigh.weight(weigh.exponent(z));
          all += a;
          n += stays && a >= set.least ? a : 0;
        }
      }
      add_soft(x);
    }, end);
  }
  if constexpr (kSoft) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) soft += __shfl_xor(soft, d, 64);
  }
  all = wave_sum64(all);
  if (lane == 0) {
    put<kOthers>(&sums->all, all);
    put<kOthers>((uint64_t*)&sums->soft, __builtin_bit_cast(uint64_t, soft));
  }
}
template <bool kOthers, class T>
__device__ __forceinline__ void sum_parts(const Row<T>& row, int w, const Settings& set, const Weigher& weigh, const Stay& stay, bool want_soft, uint64_t* part,
                                          WaveSums* sums) {
  if (want_soft && (set.greedy || set.temperature != 1.f)) sum_parts<kOthers, true>(row, w, set, weigh, stay, false, part, sums);
  else sum_parts<kOthers, false>(row, w, set, weigh, stay, want_soft, part, sums);
}

// draw, from the parts' sums and the wavefronts' in LDS (behind a barrier)
template <class T>
__device__ __forceinline__ void draw_row(const SampleArgs& a, int64_t r, const Row<T>& row, const Settings& set, const Weigher& weigh, const Stay& stay, int waves,
                                         uint32_t word, Shared& sm) {
  constexpr int kE = Row<T>::kE;
  const int lane = threadIdx.x & 63;
  uint64_t before, total;
  auto target_of = [&](uint64_t sum) { return set.greedy ? 0 : share_of(word, sum); };
  const int part = block_find([&](int i) { return sm.part[i]; }, row.parts, target_of, &before, &total, sm);
  const uint64_t target = target_of(total);
  if (threadIdx.x >= 64) return;
  typename Row<T>::Vector x[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) row.load((part * kUnroll + u) * 64 + lane, x[u]);
  // while they arrive
  uint64_t all = 0;
  double soft = 0.0;
  for (int w = lane; w < waves; w += 64) {
    all += sm.sums[w].all;
    soft += sm.sums[w].soft;
  }
  all = wave_sum64(all);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) soft += __shfl_xor(soft, d, 64);
  if (!set.greedy && set.temperature == 1.f) soft = (double)all * (1.0 / (double)kOne);
  const double log_soft = a.logp ? log(soft) : 0.0;
#pragma unroll 1
  for (int u = 0; u < kUnroll; ++u) {
    const int j = (part * kUnroll + u) * 64 + lane;
    uint64_t w[kE], sum = 0;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const float z = Row<T>::value(x[0].e[i]);
      if (set.greedy) {
        w[i] = z >= weigh.max;
      } else {
        const uint64_t weight = weigh.weight(weigh.exponent(z));
        w[i] = stay.has(key_of(z), j * kE - row.lead + i) && weight >= set.least ? weight : 0;
      }
      sum += w[i];
    }
    const uint64_t incl = wave_scan64(sum);
    uint64_t at = before + incl - sum;
    const bool mine = sum && at <= target && target < at + sum;
    if (mine) {
      Drawn d{-1, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        if (d.index < 0 && target < at + w[i]) d = Drawn{j * kE - row.lead + i, key_of(Row<T>::value(x[0].e[i])), set.greedy ? 1 : w[i], set.greedy ? 1 : total};
        at += w[i];
      }
      write_out(a, r, d, weigh, log_soft);
    }
    if (__any(mine)) return;
    before += __shfl((unsigned long long)incl, 63, 64);
#pragma unroll
    for (int v = 0; v + 1 < kUnroll; ++v) x[v].q = x[v + 1].q;
  }
}

// A workgroup per row
template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_row_kernel(SampleArgs a) {
  __shared__ Shared sm;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = blockIdx.x;
  const Row<T> row(a, r, kWaves);
  sm.powers.fill();
  const uint32_t mine = largest_key(row, wave);
  if (lane == 0) sm.top[wave] = mine;
  for (int i = threadIdx.x; i < kBins; i += kThreads) sm.hist[i] = 0;
  if (threadIdx.x == 0) sm.list_n = 0;
  __syncthreads();
  uint32_t top = 0;
  for (int w = 0; w < kWaves; ++w) top = sm.top[w] > top ? sm.top[w] : top;
  if (top <= kKeyMinusInf) {
    if (threadIdx.x == 0) nothing_to_draw(a, r);
    return;
  }
  const Settings set(a, r);
  const Weigher weigh(top, set.temperature, sm.powers);
  Stay stay{kKeyMinusInf, -1};
  if (set.ranked) {
    bin_parts(row, wave, set, weigh, sm.hist);
    __syncthreads();
    const Gather g = choose_bins(set, sm.hist, sm);
    list_parts(row, wave, weigh, g, sm.list, &sm.list_n);
    __syncthreads();
    stay = sm.list_n > kList ? threshold_slowly(row, set, weigh, top, sm) : threshold_of_list(set, weigh, top, g, (int)sm.list_n, sm);
    __syncthreads();
  }
  sum_parts<false>(row, wave, set, weigh, stay, a.logp != nullptr, sm.part, &sm.sums[wave]);
  __syncthreads();
  draw_row(a, r, row, set, weigh, stay, kWaves, a.random[r], sm);
}

// Several workgroups per row: what passes between them, in the workspace
struct RowSpace {
  uint64_t *hist, *part;
  WaveSums* sums;
  Gather* gather;
  Stay* stay;
  uint32_t *top, *count;         // count: workgroups that are done with bins, list, sums; tokens of the list
  Listed* list;
};
__host__ __device__ inline size_t row_space(char* p, int parts, int waves, RowSpace* s) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = p ? p + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  s->hist = (uint64_t*)take(kBins * 8);
  s->part = (uint64_t*)take((size_t)parts * 8);
  s->sums = (WaveSums*)take((size_t)waves * sizeof(WaveSums));
  s->gather = (Gather*)take(sizeof(Gather));
  s->stay = (Stay*)take(sizeof(Stay));
  s->top = (uint32_t*)take((size_t)waves * 4);
  s->count = (uint32_t*)take(4 * 4);
  s->list = (Listed*)take(kList * sizeof(Listed));
  return at;
}

__device__ __forceinline__ uint32_t top_of_waves(const uint32_t* tops, int waves) {
  uint32_t top = 0;
  for (int i = threadIdx.x & 63; i < waves; i += 64) top = tops[i] > top ? tops[i] : top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d, 64);
    top = o > top ? o : top;
  }
  return __builtin_amdgcn_readfirstlane(top);
}

// What this workgroup wrote is seen by the one for which this is true: the last of the row's `n`.  Every wavefront waits until its own stores have arrived in
// the L2, then one thread's fences do for all: at the scope of the whole GPU a fence writes an XCD's L2 back, or invalidates it.
__device__ __forceinline__ bool last_of_row(uint32_t* count, int n, Shared& sm) {
  __builtin_amdgcn_s_waitcnt(0x0f70);        // vmcnt(0)
  __syncthreads();
  if (threadIdx.x == 0) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    sm.last_one = atomicAdd(count, 1u) == (uint32_t)n - 1;
    if (sm.last_one) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  }
  __syncthreads();
  return sm.last_one;
}

template <class T>
struct SplitRow {
  int64_t r;
  int w, waves;
  Row<T> row;
  RowSpace s;
  __device__ __forceinline__ SplitRow(const SampleArgs& a)
      : r(blockIdx.x / a.splits), w(__builtin_amdgcn_readfirstlane((int)(blockIdx.x % a.splits) * kWaves + (threadIdx.x >> 6))), waves(a.splits * kWaves),
        row(a, r, waves) {
    row_space(a.ws + r * a.ws_row, row.parts, waves, &s);
  }
};

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_top_kernel(SampleArgs a) {
  const SplitRow<T> x(a);
  if (blockIdx.x % a.splits == 0) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) x.s.hist[i] = 0;
    if (threadIdx.x < 4) x.s.count[threadIdx.x] = 0;
  }
  const uint32_t top = largest_key(x.row, x.w);
  if ((threadIdx.x & 63) == 0) x.s.top[x.w] = top;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_bins_kernel(SampleArgs a) {
  __shared__ Shared sm;
  const SplitRow<T> x(a);
  const uint32_t top = top_of_waves(x.s.top, x.waves);
  const Settings set(a, x.r);
  if (!set.ranked || top <= kKeyMinusInf) return;
  const Weigher weigh(top, set.temperature, sm.powers);
  for (int i = threadIdx.x; i < kBins; i += kThreads) sm.hist[i] = 0;
  sm.powers.fill();
  __syncthreads();
  bin_parts(x.row, x.w, set, weigh, sm.hist);
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads)
    if (sm.hist[i]) atomicAdd((unsigned long long*)&x.s.hist[i], (unsigned long long)sm.hist[i]);
  if (!last_of_row(&x.s.count[0], a.splits, sm)) return;
  for (int i = threadIdx.x; i < kBins; i += kThreads) sm.hist[i] = __hip_atomic_load(&x.s.hist[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const Gather g = choose_bins(set, sm.hist, sm);
  if (threadIdx.x == 0) *x.s.gather = g;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_list_kernel(SampleArgs a) {
  __shared__ Shared sm;
  const SplitRow<T> x(a);
  // all loads at once, in front of the first that decides anything
  const Gather g = *x.s.gather;
  const uint32_t top = top_of_waves(x.s.top, x.waves);
  const Settings set(a, x.r);
  if (threadIdx.x == 0) sm.list_n = 0;
  if (!set.ranked || top <= kKeyMinusInf) return;
  const Weigher weigh(top, set.temperature, sm.powers);
  __syncthreads();
  list_parts(x.row, x.w, weigh, g, sm.list, &sm.list_n);
  __syncthreads();
  // one place in the row's list for all of them: places of their own for every wavefront's tokens are atomics one after another
  const int here = sm.list_n;
  if (here > 0) {
    if (threadIdx.x == 0) sm.found = atomicAdd(&x.s.count[3], (uint32_t)here);
    __syncthreads();
    for (int i = threadIdx.x; i < here && i < kList; i += kThreads) {
      const uint32_t at = sm.found + i;
      if (at < kList) put<true>((uint64_t*)&x.s.list[at], __builtin_bit_cast(uint64_t, sm.list[i]));
    }
  }
  if (!last_of_row(&x.s.count[1], a.splits, sm)) return;
  // loads of what a short list has, together with that of its length
  const Listed mine = x.s.list[threadIdx.x];
  const uint32_t n = __hip_atomic_load(&x.s.count[3], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sm.powers.fill();
  sm.list[threadIdx.x] = mine;
  if (n <= kList) {
    for (int i = threadIdx.x + kThreads; i < (int)n; i += kThreads) sm.list[i] = x.s.list[i];
  }
  __syncthreads();
  const Stay stay = n > kList ? threshold_slowly(x.row, set, weigh, top, sm) : threshold_of_list(set, weigh, top, g, (int)n, sm);
  if (threadIdx.x == 0) *x.s.stay = stay;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 4) sample_sums_kernel(SampleArgs a) {
  __shared__ Shared sm;
  const SplitRow<T> x(a);
  const Stay ranked = *x.s.stay;             // of rows without a rank anything
  const uint32_t top = top_of_waves(x.s.top, x.waves), word = a.random[x.r];
  const Settings set(a, x.r);
  if (top <= kKeyMinusInf) {
    if (blockIdx.x % a.splits == 0 && threadIdx.x == 0) nothing_to_draw(a, x.r);
    return;
  }
  const Weigher weigh(top, set.temperature, sm.powers);
  const Stay stay = set.ranked ? ranked : Stay{kKeyMinusInf, -1};
  sm.powers.fill();
  __syncthreads();
  sum_parts<true>(x.row, x.w, set, weigh, stay, a.logp != nullptr, x.s.part, &x.s.sums[x.w]);
  if (!last_of_row(&x.s.count[2], a.splits, sm)) return;
  for (int i = threadIdx.x; i < x.waves; i += kThreads) sm.sums[i] = x.s.sums[i];
  for (int i = threadIdx.x; i < x.row.parts; i += kThreads) sm.part[i] = x.s.part[i];
  __syncthreads();
  draw_row(a, x.r, x.row, set, weigh, stay, x.waves, word, sm);
}

// Workgroups per row: for every compute unit one in all, each with 4096 elements at least (one sweep of its loads), and only where that takes kWorthSplitting elements
// off a workgroup: the further launches and fences take as long.  In us without and with top-k and top-p, bf16, one workgroup per row against several: 4 rows of 32000
// 16, 29 against 19, 28 (8 each), of 50257 20, 43 against 17, 30 (12); of 152064 42, 91 against 17, 32 (32); 128 rows of 50257 21, 44 against 23, 51 (2), of 152064 46, 96 against
// 37, 81.  Two workgroups per compute unit: 200 rows of 152064 60, 134, one per row 48, 101.
constexpr int64_t kWorthSplitting = 40000;
int splits_of(int64_t n_rows, int64_t V) {
  int64_t s = 256 / n_rows;
  if (s > V / 4096) s = V / 4096;
  if (s > kMaxSplits) s = kMaxSplits;
  return s < 1 || V - V / s < kWorthSplitting ? 1 : (int)s;
}
// of a row that starts anywhere in its first vector
size_t row_bytes_of(int32_t V, int elem, int splits) {
  const int64_t e = 16 / elem, vectors = (V + (e - 1) + e - 1) / e, waves = splits * kWaves, per = 64 * kUnroll * waves;
  RowSpace s;
  return row_space(nullptr, (int)((vectors + per - 1) / per * waves), (int)waves, &s);
}

template <class T>
void launch(SampleArgs a, int32_t n_rows, hipStream_t s) {
  if (a.splits == 1) {
    constexpr int32_t kMost = kMaxWorkItems / kThreads;          // rows of a launch
    auto skip = [](auto*& p, int64_t n) { p = p ? p + n : p; };
    for (;;) {
      sample_row_kernel<T><<<n_rows < kMost ? n_rows : kMost, kThreads, 0, s>>>(a);
      if (n_rows <= kMost) return;
      n_rows -= kMost;
      a.logits = (const T*)a.logits + kMost * a.row_stride;
      skip(a.random, kMost);
      skip(a.temperature, kMost);
      skip(a.top_p, kMost);
      skip(a.min_p, kMost);
      skip(a.top_k, kMost);
      skip(a.ids, kMost);
      skip(a.logp, kMost);
      skip(a.logq, kMost);
    }
  }
  sample_top_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
  if (a.top_k || a.top_p) {
    sample_bins_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
    sample_list_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
  }
  sample_sums_kernel<T><<<n_rows * a.splits, kThreads, 0, s>>>(a);
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
