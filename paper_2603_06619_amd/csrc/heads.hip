// Norms of queries and keys, head by head, and their rotation by position, in one pass over the rows, and the gradients of both.
//
// A head's D elements lie in D / 16 lanes, two chunks of 8 elements each: of the R elements that turn, lane c has chunks c and c + R / 16, so that both elements
// of a pair (i, i + R / 2) are its own, and pairs of neighbours are anyway.  The R / 2 sines and cosines of a row are formed by a lane each and go to all heads of the
// row through LDS: a wavefront takes whole rows, of few rows parts of them.
//
// Bound by HBM: 14.4 thousand rows of 28 + 4 heads of 128 in bf16, 212 MB, take 37.5 us, 5.7 TB/s (a copy: 5.0); 20.6 thousand of 32 + 8 forward 65 us (377 MB), backward 107 (566 MB; 97 where
// the forward pass has not just read the rows past the caches) and 5 for the weights' gradients.  64 rows of 32 + 8, the step of a decoding batch, 3.7 us (6.1 with a wavefront per row).
#include "nat_internal.h"
#include "mfma_tile.hip.h"

#include <type_traits>

namespace nat {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kWaves = 4;                 // per workgroup

struct HeadsArgs {
  const void *q, *k, *wq, *wk, *dq_out, *dk_out;
  void *q_out, *k_out;                    // forward: results; backward: gradients
  const int32_t* pos;
  const double* freq;
  float* part;                            // backward: [workgroups][2][D]
  int hq, heads, turning, interleaved;    // heads: of queries and keys; turning: lanes of a head whose elements turn, R / 16
  int parts;                              // forward: wavefronts per row
  float eps;
  int64_t n_rows, q_stride, k_stride, q_out_stride, k_out_stride, dq_stride, dk_stride;
};

// 8 elements as they lie in memory.  kOnce: past the caches, for rows that nobody reads again soon.  Only where a load or store of a wavefront covers whole lines of 128 bytes, as the
// two of a head of 128 elements in bf16 do; others (heads of 64, fp32) lose by it, up to a third.
template <typename T> struct Chunk;
template <>
struct Chunk<uint16_t> {
  u32x4 x;
  template <bool kOnce = false>
  __device__ __forceinline__ static Chunk load(const uint16_t* p) { return {kOnce ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p}; }
  __device__ __forceinline__ static Chunk all(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v) >> 16;
    return {u32x4{1, 1, 1, 1} * (b | b << 16)};
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, x[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, x[i] & 0xffff0000u);
    }
  }
  template <bool kOnce = false>
  __device__ __forceinline__ static void store(uint16_t* p, const float (&v)[8]) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)v[i];
    if constexpr (kOnce) __builtin_nontemporal_store(y, (bf16x8*)p);
    else *(bf16x8*)p = y;
  }
  __device__ __forceinline__ static Chunk pick(bool a, const Chunk& p, const Chunk& q) {
    Chunk r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.x[i] = a ? p.x[i] : q.x[i];
    return r;
  }
};
template <>
struct Chunk<float> {
  f32x4 x, y;
  template <bool kOnce = false>
  __device__ __forceinline__ static Chunk load(const float* p) { return {*(const f32x4*)p, *(const f32x4*)(p + 4)}; }
  __device__ __forceinline__ static Chunk all(float v) { return {f32x4{v, v, v, v}, f32x4{v, v, v, v}}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = x[i];
      v[4 + i] = y[i];
    }
  }
  template <bool kOnce = false>
  __device__ __forceinline__ static void store(float* p, const float (&v)[8]) {
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
  __device__ __forceinline__ static Chunk pick(bool a, const Chunk& p, const Chunk& q) {
    Chunk r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.x[i] = a ? p.x[i] : q.x[i];
      r.y[i] = a ? p.y[i] : q.y[i];
    }
    return r;
  }
};

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, true));
}
// over the D / 16 lanes of a head (8 or 4, neighbours); all of them get it
template <int D>
__device__ __forceinline__ float sum_of_head(float x) {
  x += dpp<0xb1>(x);                               // lane ^ 1
  x += dpp<0x4e>(x);                               // lane ^ 2
  if constexpr (D == 128) x += dpp<0x141>(x);      // lane ^ 7, of equal fours: as lane ^ 4
  return x;
}
// over the lanes that have the same place in their heads
template <int D>
__device__ __forceinline__ float sum_of_heads(float x) {
  if constexpr (D == 64) x += dpp<0x124>(x);       // 4 and 8 lanes round in rows of 16
  x += dpp<0x128>(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return sum_halves(__builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]));
}

// What a lane is in its head, and the row's angles.
template <int D>
struct Lane {
  static constexpr int kLanes = D / 16, kHeads = 64 / kLanes;         // lanes per head, heads per step of a wavefront
  int head, at[2], angle[2];      // place of the first element of its two chunks; first angle of each (interleaved: 4 each, else 8 from angle[0])
  bool turns;
  __device__ __forceinline__ Lane(const HeadsArgs& a, int lane) {
    const int c = lane % kLanes, n = a.turning;
    head = lane / kLanes;
    turns = c < n;
    at[0] = 8 * (turns ? c : 2 * n + 2 * (c - n));
    at[1] = 8 * (turns ? c + n : 2 * n + 2 * (c - n) + 1);
    angle[0] = turns ? (a.interleaved ? 4 * c : 8 * c) : 0;
    angle[1] = turns ? (a.interleaved ? 4 * (c + n) : 8 * c + 4) : 0;
  }
};

// Sine and cosine of the row's angles, one per lane.  Of the turns, position * frequency / 2 pi, only the fraction counts: turns per position are taken as a sum of two numbers of 64 bits, good to 2^-105,
// and the product's whole turns leave it before it is rounded, so that the fraction is good to 2^-52 as long as there are fewer than 2^52 turns.  To fp32, for the functions, it is rounded by up to
// 2^-26 of a turn.
__device__ __forceinline__ void form_angles(f32x2* angles, const double* freq, int n, int pos, int lane) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (lane < n) {
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;         // 1 / 2 pi
    const double f = freq[lane], per = f * kTurn, rest = fma(f, kTurnRest, fma(f, kTurn, -per));
    const double whole = rint((double)pos * per);
    const float t = (float)fma((double)pos, rest, fma((double)pos, per, -whole));
    float s, c;
    sincospif(2.f * t, &s, &c);
    angles[lane] = f32x2{c, s};
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

struct Turn { f32x4 cs[4]; };            // (cos, sin) of the lane's 8 angles
template <int D>
__device__ __forceinline__ Turn angles_of(const f32x2* angles, const Lane<D>& l) {
  Turn t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t.cs[i] = *(const f32x4*)(angles + l.angle[i >> 1] + 2 * (i & 1));
  return t;
}

// The pairs of the two chunks by their angles, or (backward) by minus these.
template <bool kBack>
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const Turn& t, bool interleaved) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = t.cs[i >> 1][2 * (i & 1)], s = kBack ? -t.cs[i >> 1][2 * (i & 1) + 1] : t.cs[i >> 1][2 * (i & 1) + 1];
    if (interleaved) {
      float& a = i < 4 ? x[2 * i] : y[2 * i - 8];
      float& b = i < 4 ? x[2 * i + 1] : y[2 * i - 7];
      const float a0 = a;
      a = a0 * c - b * s;
      b = b * c + a0 * s;
    } else {
      const float a0 = x[i];
      x[i] = a0 * c - y[i] * s;
      y[i] = y[i] * c + a0 * s;
    }
  }
}

// 1 / sqrt(mean x^2 + eps) as a product r * s: where the root's argument passes fp32's range, x s with s = 2^-80 takes the place of x.  The sum of 128 squares of elements below 2^128 then stays below
// 2^103; as it comes from a mean of 2^103 on, what falls out of the range below has no weight.
template <int D>
__device__ __forceinline__ void norm_of(const float (&x)[8], const float (&y)[8], float eps, float* r, float* s) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
  float mean = fmaf(sum_of_head<D>(sum), 1.f / D, eps);
  *s = 1.f;
  if (__any(mean == INFINITY)) {
    const float z = mean == INFINITY ? 0x1p-80f : 1.f;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = fmaf(x[i] * z, x[i] * z, fmaf(y[i] * z, y[i] * z, t));
    mean = fmaf(sum_of_head<D>(t), 1.f / D, eps * z * z);          // (z * z alone would be zero)
    *s = z;
  }
  *r = rsqrtf(mean);
}

// Inputs are read past the caches, which the results fill for the next launch: 20.6 thousand rows of 32 + 8 heads 63 us, otherwise 77, between launches that write the inputs and read the
// results 222 and 227, 14.4 thousand of 28 + 4 115 and 124.  (Results past the caches: 79 instead of 71 with the launch that reads them.)
// Without loads ahead: 83 registers, five wavefronts per SIMD.  With them, as in the backward pass, 102 and four: 14.4 thousand rows of 28 + 4 heads 36 instead of 33 us.
template <typename T, int D>
__global__ void __launch_bounds__(64 * kWaves) heads_fwd_kernel(HeadsArgs a) {
  constexpr bool kOnce = D == 128 && sizeof(T) == 2;
  __shared__ __attribute__((aligned(16))) f32x2 angles[kWaves][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane<D> l(a, lane);
  const Chunk<T> one = Chunk<T>::all(1.f);
  Chunk<T> wq[2] = {one, one}, wk[2] = {one, one};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (a.wq) wq[i] = Chunk<T>::load((const T*)a.wq + l.at[i]);
    if (a.wk) wk[i] = Chunk<T>::load((const T*)a.wk + l.at[i]);
  }
  for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < a.n_rows * a.parts; unit += (int64_t)gridDim.x * kWaves) {
    const int64_t row = a.parts == 1 ? unit : unit / a.parts;
    const int part = (int)(unit - row * a.parts);
    Turn t = {};
    if (a.turning) {
      form_angles(angles[wave], a.freq, 8 * a.turning, a.pos[row], lane);
      t = angles_of<D>(angles[wave], l);
    }
    for (int h = part * Lane<D>::kHeads + l.head; h < a.heads; h += a.parts * Lane<D>::kHeads) {
      const bool is_q = h < a.hq;
      const T* from = is_q ? (const T*)a.q + row * a.q_stride + h * D : (const T*)a.k + row * a.k_stride + (h - a.hq) * D;
      T* to = is_q ? (T*)a.q_out + row * a.q_out_stride + h * D : (T*)a.k_out + row * a.k_out_stride + (h - a.hq) * D;
      float x[8], y[8], w[8];
      Chunk<T>::template load<kOnce>(from + l.at[0]).get(x);
      Chunk<T>::template load<kOnce>(from + l.at[1]).get(y);
      if (is_q ? a.wq != nullptr : a.wk != nullptr) {
        float r, s;
        norm_of<D>(x, y, a.eps, &r, &s);
        Chunk<T>::pick(is_q, wq[0], wk[0]).get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * s * r * w[i];
        Chunk<T>::pick(is_q, wq[1], wk[1]).get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * s * r * w[i];
      }
      if (l.turns) turn<false>(x, y, t, a.interleaved);
      Chunk<T>::store(to + l.at[0], x);
      Chunk<T>::store(to + l.at[1], y);
    }
  }
}

// Steps of a wavefront through a row: the queries' heads, then the keys', kHeads at a time.  What the next step needs is loaded before this one's is worked on, without a branch
// around the loads (behind one the compiler waits for all of them): places that are not there are others of the same array, whose values go nowhere.
struct Steps {
  int q, all;                            // of queries, and of both
  template <int D>
  __device__ __forceinline__ static Steps of(const HeadsArgs& a) {
    constexpr int n = Lane<D>::kHeads;
    const int q = (a.hq + n - 1) / n;
    return {q, q + (a.heads - a.hq + n - 1) / n};
  }
};
template <typename T, int D>
__device__ __forceinline__ const T* element_of(const HeadsArgs& a, const Steps& steps, int64_t row, int step, const Lane<D>& l, const void* q, const void* k, int64_t q_stride,
                                               int64_t k_stride) {
  const bool is_q = step < steps.q;
  const int heads = is_q ? a.hq : a.heads - a.hq, h = (is_q ? step : step - steps.q) * Lane<D>::kHeads + l.head;
  return (is_q ? (const T*)q + row * q_stride : (const T*)k + row * k_stride) + (h < heads ? h : heads - 1) * D;
}

template <typename T>
struct Pair {
  Chunk<T> x, y;
  template <bool kOnce = false>
  __device__ __forceinline__ static Pair load(const T* p, const int (&at)[2]) {
    return {Chunk<T>::template load<kOnce>(p + at[0]), Chunk<T>::template load<kOnce>(p + at[1])};
  }
};

// A lane adds up the weights' gradients of its elements over its rows and heads; its workgroup's sums go to `part`.  Three wavefronts per SIMD; loads a step ahead took 20.6 thousand
// rows of 32 + 8 heads from 122 to 117 us, and 2940 of 16 + 16 heads of 64 in fp32, for which there is hardly a second row per wavefront, from 25.5 to 18.3 (with sums across
// lanes by DPP and lane swaps).
template <typename T, int D, bool kOnce>
__global__ void __launch_bounds__(64 * kWaves) heads_bwd_kernel(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) f32x2 angles[kWaves][D / 2];
  __shared__ __attribute__((aligned(16))) float sums[kWaves][2][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane<D> l(a, lane);
  const Steps steps = Steps::of<D>(a);
  const int64_t stride = (int64_t)gridDim.x * kWaves, first = (int64_t)blockIdx.x * kWaves + wave;
  float dw[2][16] = {};                  // of queries and keys
  if (first < a.n_rows) {
    struct Both { Pair<T> x, g; };
    auto load = [&](int64_t row, int step) __attribute__((always_inline)) {
      return Both{Pair<T>::template load<kOnce>(element_of<T, D>(a, steps, row, step, l, a.q, a.k, a.q_stride, a.k_stride), l.at),
                  Pair<T>::template load<kOnce>(element_of<T, D>(a, steps, row, step, l, a.dq_out, a.dk_out, a.q_out_stride, a.k_out_stride), l.at)};
    };
    Both next = load(first, 0);
    int next_pos = a.turning ? a.pos[first] : 0;
    const Pair<T> one = {Chunk<T>::all(1.f), Chunk<T>::all(1.f)};
    const Pair<T> weights[2] = {a.wq ? Pair<T>::load((const T*)a.wq, l.at) : one, a.wk ? Pair<T>::load((const T*)a.wk, l.at) : one};
    for (int64_t row = first; row < a.n_rows; row += stride) {
      const int64_t row1 = row + stride < a.n_rows ? row + stride : row;
      Turn t = {};
      if (a.turning) {
        form_angles(angles[wave], a.freq, 8 * a.turning, next_pos, lane);
        next_pos = a.pos[row1];
        t = angles_of<D>(angles[wave], l);
      }
      auto side = [&](auto is_k) __attribute__((always_inline)) {
        constexpr bool kKeys = decltype(is_k)::value;
        const bool norm = kKeys ? a.wk != nullptr : a.wq != nullptr;
        const int begin = kKeys ? steps.q : 0, end = kKeys ? steps.all : steps.q, heads = kKeys ? a.heads - a.hq : a.hq;
        T* out = kKeys ? (T*)a.k_out + row * a.dk_stride : (T*)a.q_out + row * a.dq_stride;
        for (int step = begin; step < end; ++step) {
          const Both raw = next;
          const bool more = !kKeys || step + 1 < end;
          next = load(more ? row : row1, more ? step + 1 : 0);
          const int h = (step - begin) * Lane<D>::kHeads + l.head;
          float g0[8], g1[8];
          raw.g.x.get(g0);
          raw.g.y.get(g1);
          if (l.turns) turn<true>(g0, g1, t, a.interleaved);
          if (norm) {
            float x[8], y[8], w[8], r, s, dot = 0.f;
            raw.x.x.get(x);
            raw.x.y.get(y);
            norm_of<D>(x, y, a.eps, &r, &s);
            const float rs = r * s;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              x[i] = x[i] * s * r;               // of norm sqrt(D), almost
              y[i] = y[i] * s * r;
            }
            if (h < heads) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                dw[kKeys][i] = fmaf(g0[i], x[i], dw[kKeys][i]);
                dw[kKeys][8 + i] = fmaf(g1[i], y[i], dw[kKeys][8 + i]);
              }
            }
            weights[kKeys].x.get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              g0[i] *= w[i];
              dot = fmaf(g0[i], x[i], dot);
            }
            weights[kKeys].y.get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              g1[i] *= w[i];
              dot = fmaf(g1[i], y[i], dot);
            }
            dot = sum_of_head<D>(dot) * (1.f / D);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              g0[i] = rs * (g0[i] - x[i] * dot);
              g1[i] = rs * (g1[i] - y[i] * dot);
            }
          }
          if (h < heads) {
            Chunk<T>::template store<kOnce>(out + h * D + l.at[0], g0);
            Chunk<T>::template store<kOnce>(out + h * D + l.at[1], g1);
          }
        }
      };
      side(std::false_type{});
      side(std::true_type{});
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = sum_of_heads<D>(dw[s][i]);
      if (l.head == 0) sums[wave][s][l.at[i >> 3] + (i & 7)] = x;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += 64 * kWaves) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += (&sums[w][0][0])[i];
    a.part[(int64_t)blockIdx.x * 2 * D + i] = x;
  }
}

// The workgroups' sums in order: one workgroup per kColumns elements, every kWalkers-th part to each walker, eight loads ahead (768 parts 4 us; one after the other 48).
constexpr int kColumns = 8, kWalkers = 256 / kColumns;
__global__ void __launch_bounds__(256) heads_weights_kernel(const float* part, int n_parts, int D, float* dwq, float* dwk, int accumulate) {
  __shared__ float sums[kWalkers][kColumns + 1];
  const int column = threadIdx.x % kColumns, walker = threadIdx.x / kColumns, e = blockIdx.x * kColumns + column;
  float x = 0.f;
  for (int i0 = walker; i0 < n_parts; i0 += 8 * kWalkers) {
    float y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) y[u] = i0 + u * kWalkers < n_parts ? part[(int64_t)(i0 + u * kWalkers) * 2 * D + e] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) x += y[u];
  }
  sums[walker][column] = x;
  __syncthreads();
  if (walker) return;
  x = 0.f;
#pragma unroll
  for (int w = 0; w < kWalkers; ++w) x += sums[w][column];
  float* to = e < D ? dwq : dwk;
  if (!to) return;
  to += e < D ? e : e - D;
  *to = accumulate ? *to + x : x;
}

bool misaligned(const void* p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

// results in the place of the inputs, but in other rows
bool other_rows(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t n_rows) {
  return n_rows > 1 && in != nullptr && in == out && in_stride != out_stride;
}

// Gradients of more than it holds go past the caches both ways: 20.6 thousand rows of 32 + 8 heads 97 us, kept 117, between launches that write the gradients and read the results 348 and
// 363; 5.8 thousand, 177 MB, between such launches 193 and 190.
constexpr int64_t kInfinityCache = 256 << 20;
constexpr int kMostBlocks = 1280, kMostSums = 768;       // as many as fit at once, or nearly; backward each leaves sums
int blocks_of(int64_t n_rows, int most) {
  const int64_t n = (n_rows + kWaves - 1) / kWaves;
  return (int)(n < 1 ? 1 : n < most ? n : most);
}

nat_status heads_args(const nat_qk_params* p, const void* d_q, const void* d_k, const void* d_q_weight, const void* d_k_weight,
                      const int32_t* d_position_ids, const double* d_inv_freq, HeadsArgs* a) {
  if (!p || p->n_rows < 0 || p->n_rows > INT32_MAX || !(p->eps > 0.f) || !(p->eps < INFINITY) || (p->interleaved & ~1)) return NAT_INVALID_ARG;
  if (p->dtype != NAT_DTYPE_BF16 && p->dtype != NAT_DTYPE_F32) return NAT_UNSUPPORTED_DTYPE;
  const int D = p->head_dim;
  if ((D != 64 && D != 128) || p->n_q_heads < 1 || p->n_q_heads > 4096 || p->n_kv_heads < 1 || p->n_kv_heads > 4096 || p->rotary_dim < 0 ||
      p->rotary_dim > D || p->rotary_dim % 16)
    return NAT_BAD_SHAPE;
  const int64_t row[2] = {(int64_t)p->n_q_heads * D, (int64_t)p->n_kv_heads * D};
  const int64_t* strides[6] = {&p->q_stride, &p->k_stride, &p->q_out_stride, &p->k_out_stride, &p->dq_stride, &p->dk_stride};
  int64_t* to[6] = {&a->q_stride, &a->k_stride, &a->q_out_stride, &a->k_out_stride, &a->dq_stride, &a->dk_stride};
  for (int i = 0; i < 6; ++i) {
    const int64_t s = *strides[i];
    if (s != 0 && (s < row[i & 1] || s % (p->dtype == NAT_DTYPE_BF16 ? 8 : 4) || s > INT32_MAX)) return NAT_BAD_SHAPE;
    *to[i] = s ? s : row[i & 1];
  }
  if (misaligned(d_q) || misaligned(d_k) || misaligned(d_q_weight) || misaligned(d_k_weight) || misaligned(d_inv_freq, 8)) return NAT_INVALID_ARG;
  if (p->n_rows > 0 && (!d_q || !d_k || (p->rotary_dim > 0) != (d_position_ids != nullptr) || (p->rotary_dim > 0 && !d_inv_freq))) return NAT_INVALID_ARG;
  a->q = d_q;
  a->k = d_k;
  a->wq = d_q_weight;
  a->wk = d_k_weight;
  a->pos = d_position_ids;
  a->freq = d_inv_freq;
  a->hq = p->n_q_heads;
  a->heads = p->n_q_heads + p->n_kv_heads;
  a->turning = p->rotary_dim / 16;
  a->interleaved = p->interleaved;
  a->eps = p->eps;
  a->n_rows = p->n_rows;
  return NAT_OK;
}

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" nat_status nat_qk_norm_rope(const nat_qk_params* params, const void* d_q, const void* d_k, const void* d_q_weight, const void* d_k_weight,
                                       const int32_t* d_position_ids, const double* d_inv_freq, void* d_q_out, void* d_k_out, void* stream) {
  HeadsArgs a{};
  const nat_status st = heads_args(params, d_q, d_k, d_q_weight, d_k_weight, d_position_ids, d_inv_freq, &a);
  if (st != NAT_OK) return st;
  if (misaligned(d_q_out) || misaligned(d_k_out) || other_rows(d_q, a.q_stride, d_q_out, a.q_out_stride, a.n_rows) ||
      other_rows(d_k, a.k_stride, d_k_out, a.k_out_stride, a.n_rows))
    return NAT_INVALID_ARG;
  if (a.n_rows == 0) return NAT_OK;
  if (!d_q_out || !d_k_out) return NAT_INVALID_ARG;
  a.q_out = d_q_out;
  a.k_out = d_k_out;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_HEADS, s);
  // of few rows each by several wavefronts, of up to as many steps as it has
  const int steps = (a.heads * params->head_dim + 1023) / 1024;
  const int64_t most = kMostBlocks * kWaves / a.n_rows;
  a.parts = most < 1 ? 1 : most < steps ? (int)most : steps;
  const int n = blocks_of(a.n_rows * a.parts, kMostBlocks);
  if (params->dtype == NAT_DTYPE_BF16) {
    if (params->head_dim == 128) heads_fwd_kernel<uint16_t, 128><<<n, 64 * kWaves, 0, s>>>(a);
    else heads_fwd_kernel<uint16_t, 64><<<n, 64 * kWaves, 0, s>>>(a);
  } else {
    if (params->head_dim == 128) heads_fwd_kernel<float, 128><<<n, 64 * kWaves, 0, s>>>(a);
    else heads_fwd_kernel<float, 64><<<n, 64 * kWaves, 0, s>>>(a);
  }
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}

extern "C" size_t nat_qk_norm_rope_bwd_workspace_bytes(int64_t n_rows, int32_t head_dim) {
  if (n_rows <= 0 || n_rows > INT32_MAX || (head_dim != 64 && head_dim != 128)) return 0;
  return ((size_t)blocks_of(n_rows, kMostSums) * 2 * head_dim * 4 + 255) / 256 * 256;
}

extern "C" nat_status nat_qk_norm_rope_bwd(const nat_qk_params* params, const void* d_q, const void* d_k, const void* d_q_weight, const void* d_k_weight,
                                           const int32_t* d_position_ids, const double* d_inv_freq, const void* d_dq_out, const void* d_dk_out,
                                           void* d_dq, void* d_dk, float* d_dq_weight, float* d_dk_weight, int32_t accumulate, void* d_ws,
                                           size_t ws_bytes, void* stream) {
  HeadsArgs a{};
  const nat_status st = heads_args(params, d_q, d_k, d_q_weight, d_k_weight, d_position_ids, d_inv_freq, &a);
  if (st != NAT_OK) return st;
  if (misaligned(d_dq_out) || misaligned(d_dk_out) || misaligned(d_dq) || misaligned(d_dk) || misaligned(d_dq_weight, 4) || misaligned(d_dk_weight, 4) ||
      (d_q_weight != nullptr) != (d_dq_weight != nullptr) || (d_k_weight != nullptr) != (d_dk_weight != nullptr) ||
      other_rows(d_dq_out, a.q_out_stride, d_dq, a.dq_stride, a.n_rows) || other_rows(d_dk_out, a.k_out_stride, d_dk, a.dk_stride, a.n_rows))
    return NAT_INVALID_ARG;
  const bool weights = d_q_weight || d_k_weight;
  if (a.n_rows > 0 && (!d_dq_out || !d_dk_out || !d_dq || !d_dk)) return NAT_INVALID_ARG;
  if (a.n_rows > 0 && weights && (!d_ws || ws_bytes < nat_qk_norm_rope_bwd_workspace_bytes(a.n_rows, params->head_dim))) return NAT_WORKSPACE_TOO_SMALL;
  if (misaligned(d_ws, 256)) return NAT_INVALID_ARG;
  a.dq_out = d_dq_out;
  a.dk_out = d_dk_out;
  a.q_out = d_dq;
  a.k_out = d_dk;
  a.part = weights ? (float*)d_ws : nullptr;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_HEADS, s);
  const int n = a.n_rows > 0 ? blocks_of(a.n_rows, kMostSums) : 0, D = params->head_dim;
  if (n > 0) {
    if (params->dtype == NAT_DTYPE_BF16) {
      if (D == 128 && a.n_rows * a.heads * (D * 2 * 3) > kInfinityCache) heads_bwd_kernel<uint16_t, 128, true><<<n, 64 * kWaves, 0, s>>>(a);
      else if (D == 128) heads_bwd_kernel<uint16_t, 128, false><<<n, 64 * kWaves, 0, s>>>(a);
      else heads_bwd_kernel<uint16_t, 64, false><<<n, 64 * kWaves, 0, s>>>(a);
    } else {
      if (D == 128) heads_bwd_kernel<float, 128, false><<<n, 64 * kWaves, 0, s>>>(a);
      else heads_bwd_kernel<float, 64, false><<<n, 64 * kWaves, 0, s>>>(a);
    }
    NAT_LAUNCH_CHECK();
  }
  if (weights && (n > 0 || !accumulate)) {
    heads_weights_kernel<<<2 * D / kColumns, 256, 0, s>>>(a.part, n, D, d_dq_weight, d_dk_weight, accumulate);
    NAT_LAUNCH_CHECK();
  }
  return NAT_OK;
}
