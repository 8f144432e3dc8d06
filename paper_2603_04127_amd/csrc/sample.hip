// Drawing the next token of every row from its logits: temperature, top_k, top_p, min_p, by a given random number.
//
// With w_t = exp((x_t - max x) / T) and the tokens in order of their logits (equal ones by their number), a row keeps the first top_k of them; of
// those, the shortest beginning that holds top_p of their sum; and of those the ones with w_t >= min_p.  The token drawn is the first, in
// the order of the tokens' numbers, behind which the kept weights add up to more than u times their sum.
//
// A workgroup takes a row, and reads it once for each question: the largest logit; those that top_k can keep, or the weights by bins of their logits; the
// last that top_p keeps; the sum of what is kept.  What is kept is a beginning of the order, so that its last entry says it.
//  * Small top_k: a bound from the threads' maxima leaves few candidates, which count those before them and, kept, the weights of those with
//    lower numbers: two reads of the row.
//  * Else a histogram of weights over the logits finds the bin where the beginning ends; the read that lists its entries, for them to be sorted, adds up
//    the weights before it.
//  * The draw sums the kept weights by waves, each of which holds a contiguous part of the row, and looks into one of them.  A row that keeps
//    everything has these sums from the first read.
// Weights are in fp64, by a polynomial, to 2^-33 of their value, and so are their sums; a histogram's are integers, whose sums have no order, in units that go
// with the bins.  (With one unit for all bins, of the largest weight, a long tail counted as nothing: of one token and 2^25 of 2^-37 each, top_p 0.9999 kept the one alone.)
// In fp32 the borders between a large row's tokens would be off by some 2^-30 of the row's sum each, 2^17 of them together by 2^-13: one
// row in 8000 would draw a token's neighbour.
// What bounds it: of 256 rows of 131071 bf16 logits the first read takes 10 us (6.7 TB/s), a read that asks a comparison of each logit 9, one that weighs
// each 24 (19 instructions a logit, four waves a SIMD; the matrix of 67 MB lies in the last cache by then), the histogram's 40 (two more for the
// addition in LDS and its bin).  Together: the largest alone 28 us, top_k 50 32, no filter 38 (weighed in a read of its own behind that for the largest:
// 47), top_p 0.9 105 to 107 (with a read for the list and one for the sum 6 more); one row of 32000 fp32 logits 8, 13, 13 and 30, where the way through the
// steps counts and not the row (top_k 50 with the bound's bits four at a time alone: 14.4).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace dark {
namespace sample {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMostGroups = 1 << 21;   // workgroups in one dimension of a grid: 2^31 threads, of less than 2^32
constexpr int kAhead = 4;      // pieces of 16 bytes that a thread asks for at once
constexpr int kBins = 2048;    // 32 for each lane of a wave
constexpr int kList = 2048;    // entries that are sorted
constexpr int kSmall = 512;    // the largest top_k that goes by the threads' maxima
constexpr int kCounted = 256;  // entries that count each other; more are sorted by merging

// Monotone in the value for everything but NaN; 0 is below every value.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v + 0.f);   // one zero
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

struct Setting {
  const float *temperature, *top_p, *min_p;   // of every row, or null: the call's
  const int32_t* top_k;
  float T, p, q;
  int k;
};

// The row's elements for one thread: waves have contiguous parts, lanes neighbouring pieces.
template <typename T>
struct Row {
  static constexpr int P = 16 / (int)sizeof(T);
  __amdgpu_buffer_rsrc_t at;
  int begin, V, pieces;   // token of the row's first piece's first element (it may lie before the row); tokens; pieces of a thread
  bool infinite;          // the largest logit is infinite: those that are share everything
  __device__ u32x4 ask(int piece) const { return __builtin_amdgcn_raw_buffer_load_b128(at, (unsigned)piece * 16u, 0, 0); }
  // a piece's logits: -infinity where there is no token; in a row with infinite ones these are 0 and all others -infinity
  __device__ u32x4 logits(u32x4 v, int t) const {
    if (t < 0 || t + P > V) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const bool there = (unsigned)(t + j) < (unsigned)V;
        if constexpr (sizeof(T) == 2) {
          const unsigned w = v[j / 2];
          v[j / 2] = there ? w : j & 1 ? (w & 0xffffu) | 0xff800000u : (w & 0xffff0000u) | 0xff80u;
        } else {
          v[j] = there ? v[j] : 0xff800000u;
        }
      }
    }
    if (infinite) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) v[j] = ((v[j] & 0xffffu) == 0x7f80u ? 0u : 0xff80u) | (v[j] >> 16 == 0x7f80u ? 0u : 0xff800000u);
        else v[j] = v[j] == 0x7f800000u ? 0u : 0xff800000u;
      }
    }
    return v;
  }
  __device__ u32x4 fetch(int piece) const { return logits(ask(piece), begin + piece * P); }
  __device__ int piece(int wave, int lane, int i) const { return (wave * pieces + i) * 64 + lane; }
  __device__ static float value(u32x4 v, int j) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(j & 1 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16);
    else return __uint_as_float(v[j]);
  }
  __device__ static void drop(u32x4& v, int j) {
    if constexpr (sizeof(T) == 2) v[j / 2] = j & 1 ? (v[j / 2] & 0xffffu) | 0xff800000u : (v[j / 2] & 0xffff0000u) | 0xff80u;
    else v[j] = 0xff800000u;
  }
  __device__ static float largest(u32x4 v) {
    float m = value(v, 0);
#pragma unroll
    for (int j = 1; j < P; ++j) m = fmaxf(m, value(v, j));
    return m;
  }
  // f(element, token) for a piece's elements, in a loop: for what is rarely needed, or needs many registers
  template <typename F>
  __device__ static __forceinline__ void elements(u32x4 v, int t, const F& f) {
#pragma unroll 1
    for (int j = 0; j < P; ++j) {
      f(value(v, 0), t + j);
      if constexpr (sizeof(T) == 2) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
      else v = u32x4{v[1], v[2], v[3], 0};
    }
  }
  // f(element, token) for those of a piece's elements that lie between two values
  template <typename F>
  __device__ static __forceinline__ void between(u32x4 v, int t, float from, float to, const F& f) {
    unsigned hits = 0;
#pragma unroll
    for (int j = 0; j < P; ++j) hits |= value(v, j) >= from && value(v, j) <= to ? 1u << j : 0u;
    while (hits != 0) {
      const int j = __builtin_ctz(hits), w = sizeof(T) == 2 ? j >> 1 : j;
      const unsigned word = w & 2 ? (w & 1 ? v[3] : v[2]) : (w & 1 ? v[1] : v[0]);
      f(__uint_as_float(sizeof(T) == 2 ? j & 1 ? word & 0xffff0000u : word << 16 : word), t + j);
      hits &= hits - 1;
    }
  }
  // f(piece, its first token) for the thread's pieces
  template <typename F>
  __device__ __forceinline__ void each(int wave, int lane, const F& f) const {
#pragma unroll 1
    for (int i = 0; i < pieces; i += kAhead) {
      u32x4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) v[k] = ask(piece(wave, lane, i + k));   // behind the row: nothing is read
      const int n = min(pieces - i, kAhead);
#pragma unroll 1
      for (int k = 0; k < n; ++k) {   // one copy of f: the instruction cache is to hold the kernel
        const int t = begin + piece(wave, lane, i + k) * P;
        f(logits(v[0], t), t);
#pragma unroll
        for (int j = 0; j + 1 < kAhead; ++j) v[j] = v[j + 1];
      }
    }
  }
};

// exp((x - m) / T) = 2^z = 2^n 2^f, f at most 1/2: 2^f = 1 + f g(f), g the polynomial that equals it at the seven zeros of Chebyshev's T_7; off by
// 2^-33.  Rounding to n by the constant whose last bit is a unit, and the exponent by an integer addition: conversions and ldexp of fp64 cost more.
// Only for what is not below `floor`, where z is some -1000: weights there are 0.
struct Weight {
  double m, c;     // c = log2 e / T
  float floor;
  // times 2^up
  __device__ __forceinline__ double operator()(float x, int up = 0) const {
    const double z = ((double)x - m) * c, t = z + 6755399441055744.0, f = z - (t - 6755399441055744.0);
    double y = fma(f, 1.529732376073432e-05, 1.5461444698569848e-4);
    y = fma(f, y, 1.3333502386162631e-3);
    y = fma(f, y, 9.6180566785246356e-3);
    y = fma(f, y, 5.5504108839096185e-2);
    y = fma(f, y, 2.4022650922288757e-1);
    y = fma(f, y, 6.9314718055994529e-1);
    y = fma(f, y, 1.0);
    return __hiloint2double(__double2hiint(y) + (int)((unsigned)(__double2loint(t) + up) << 20), __double2loint(y));
  }
  // the same for any logit; -infinity and NaN weigh nothing
  __device__ __forceinline__ double any(float x, int up = 0) const { return x >= floor ? (*this)(x, up) : 0.0; }
};

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_prefix(T v, int lane) {   // up to and including the lane's own
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T x = __shfl_up(v, o, 64);
    if (lane >= o) v += x;
  }
  return v;
}

// An entry of the order: the larger first.
__device__ __forceinline__ u64 entry(float x, int token) { return (u64)ordered(x) << 32 | (unsigned)~token; }
__device__ __forceinline__ float logit_of(u64 e) { return value_of((unsigned)(e >> 32)); }
__device__ __forceinline__ int token_of(u64 e) { return (int)~(unsigned)e; }

struct Shared {
  u64 list[kList];
  u64 mass[kBins];
  unsigned count[kBins];
  double sums[kWaves], scan[kWaves], weights[kSmall];
  float tops[kThreads];
  u64 bound;         // the last entry that is kept
  double before;     // weight of the bins before the chosen one
  double target;     // the weight that top_p asks for
  int ranks_before, bin, size, kept, again;
};

// The list's first n entries in descending order.
__device__ __forceinline__ void sort(Shared& s, int n, int tid) {
  if (n <= kCounted) {
    const u64 own = tid < n ? s.list[tid] : 0;
    if (tid >= n && tid < n + 8) s.list[tid] = 0;
    __syncthreads();
    int before = 0;
    if (tid < n)
      for (int i = 0; i < n; i += 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) before += s.list[i + j] > own;
    __syncthreads();
    if (tid < n) s.list[before] = own;   // entries are distinct
    __syncthreads();
    return;
  }
  int size = kCounted;
  while (size < n) size *= 2;
  for (int i = tid; i < size; i += kThreads)
    if (i >= n) s.list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int i = tid; i < size / 2; i += kThreads) {
        const int a = 2 * i - (i & (j - 1)), b = a + j;
        const u64 x = s.list[a], y = s.list[b];
        if (((a & k) == 0) == (x < y)) {
          s.list[a] = y;
          s.list[b] = x;
        }
      }
      __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(const T* __restrict__ logits, const float* __restrict__ uniform, Setting set,
                                                     int32_t* __restrict__ out_token, float* __restrict__ out_logprob, int B, int V) {
  __shared__ Shared s;
  // Bit 9 of MODE, IEEE, off: a maximum of a signalling NaN and a number is the number.
  __builtin_amdgcn_s_setreg(1 | 9 << 6, 0);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.y * kMostGroups + blockIdx.x;
  if (b >= B) return;
  constexpr int P = Row<T>::P;
  Row<T> row;
  {
    const long long first = (long long)b * V, base = first / P * P;
    const long long bytes = (first + V - base) * (long long)sizeof(T);
    row.at = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(logits + base), 0, (int)((bytes + 3) & ~3LL), 0x00027000);
    row.begin = (int)(base - first);
    row.V = V;
    const int all = (int)((first + V - base + P - 1) / P);
    row.pieces = (all + kThreads - 1) / kThreads;
  }
  row.infinite = false;
  const float temp = set.temperature != nullptr ? set.temperature[b] : set.T;
  int k = set.top_k != nullptr ? set.top_k[b] : set.k;
  float p = set.top_p != nullptr ? set.top_p[b] : set.p, q = set.min_p != nullptr ? set.min_p[b] : set.q, u = uniform != nullptr ? uniform[b] : 0.f;   // asked for before the row
  Weight weight;
  weight.c = temp > 0.f ? fmin(1.4426950408889634 / (double)temp, 1e300) : 1.0;
  const auto set_floor = [&]() __attribute__((always_inline)) {
    // rounded up: z stays where the exponent holds it; the largest logit weighs 1
    const double least = weight.m - 1000.0 / weight.c;
    weight.floor = least > -3.402823466e38 ? fminf(value_of(ordered((float)least) + 1u), (float)weight.m) : -3.402823466e38f;
  };
  // The largest logit, of every thread and of all.  A row that keeps everything is weighed on the way, beside the largest of the wave's first logits: the
  // exponent holds what is larger, up to 2^900 (else, and where those are all masked, it is weighed again).
  const bool everything = temp > 0.f && (k <= 0 || k >= V) && !(p < 1.f) && !(q > 0.f);
  float mine = -INFINITY, beside = -INFINITY;
  double sum = 0.0;
  if (everything) {
    bool first = true;
    row.each(wave, lane, [&](u32x4 v, int) __attribute__((always_inline)) {
      const float most = Row<T>::largest(v);   // of a NaN and a number: the number
      mine = fmaxf(mine, most);
      if (first) {
        first = false;
        beside = wave_max(most);
        weight.m = fabsf(beside) < INFINITY ? beside : 0.0;
        set_floor();
      }
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float x = Row<T>::value(v, j);
        const double w = weight(x);
        sum += x >= weight.floor ? w : 0.0;
        if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    });
    sum = wave_sum(sum);
  } else {
    row.each(wave, lane, [&](u32x4 v, int) __attribute__((always_inline)) { mine = fmaxf(mine, Row<T>::largest(v)); });
  }
  s.tops[tid] = mine;
  if (tid == 0) s.again = 0;
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, s.tops[i * 64 + lane]);
  top = wave_max(top);
  if (!(top > -INFINITY)) {
    if (tid == 0) {
      out_token[b] = -1;
      if (out_logprob != nullptr) out_logprob[b] = -INFINITY;
    }
    return;
  }
  if (top == INFINITY) {
    row.infinite = true;
    mine = mine == INFINITY ? 0.f : -INFINITY;
    top = 0.f;
    __syncthreads();
    s.tops[tid] = mine;
    __syncthreads();
  }
  weight.m = top;
  if (!(temp > 0.f)) {   // the largest logit
    k = 1;
    p = 1.f;
  }
  set_floor();
  q = q > 0.f ? fminf(q, 1.f) : 0.f;
  u = u > 0.f ? u : 0.f;
  if (k <= 0 || k >= V) k = 0;
  const bool by_p = p < 1.f;
  if (!(p > 0.f)) p = by_p ? 0.f : 1.f;
  u64 bound = 0;   // entries from this one on are kept
  // A histogram's weights are whole numbers, of a unit that every octave of the order has for itself: a weight of 2^-(o+1) ... 2^-o counts as 2^(bits-1) ...
  // 2^bits, so that it keeps 2^-bits of its value, 2^-34 at least, however many there are; it stays below 2^52, and V of them below 2^63.
  const int bits = min(__builtin_clz((unsigned)V) + 30, 51);
  const double unit = (double)(1ull << bits);
  const auto integer = [&](double w) __attribute__((always_inline)) -> u64 { return (u64)__double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull; };
  const auto value_in = [&](u64 sum, int octave) __attribute__((always_inline)) -> double { return (double)sum * __hiloint2double((1023 - bits - octave) << 20, 0); };

  // What the sums before a token are held against.  1 or more: whatever they are, the last token has it, though it may weigh less than their roundings.
  const auto share_of = [&](double all) __attribute__((always_inline)) -> double { return u < 1.f ? (double)u * all : INFINITY; };

  // The list holds all entries of a part of the order, sorted, behind `rank` entries of weight `held`: the last that is kept of them, by rank
  // or by weight (target; the first at least), and the weight up to it.  By one wave.
  const auto last_of = [&](int n, int rank, double held, bool by_rank, int most, double target, double* upto) __attribute__((always_inline)) -> u64 {
    u64 found = 0;
    double sum = held;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const u64 e = i0 + lane < n ? s.list[i0 + lane] : 0;
      const double up = sum + wave_prefix(e != 0 ? weight.any(logit_of(e)) : 0.0, lane), below = __shfl_up(up, 1, 64);
      const bool in = e != 0 && (by_rank ? rank + i0 + lane < most : (lane == 0 ? sum : below) < target || i0 + lane == 0);
      const u64 kept = __ballot(in);
      if (kept != 0) {
        const int last = 63 - __builtin_clzll(kept);
        found = __shfl(e, last, 64);
        *upto = __shfl(up, last, 64);
        if (lane == 0) s.kept = i0 + last + 1;
      }
      sum = __shfl(up, 63, 64);
    }
    return found;
  };
  const auto append = [&](float x, int t) __attribute__((always_inline)) {
    const int at = atomicAdd(&s.size, 1);
    if (at < kList) s.list[at] = entry(x, t);
  };
  const auto finish = [&](int token, double w, double all) __attribute__((always_inline)) {
    out_token[b] = token;
    if (out_logprob != nullptr) out_logprob[b] = (float)log(w / all);
  };

  bool summed = false;   // whether `sum` is that of a thread's weights before the bin that holds the bound, and the list's first s.kept are what is kept of it
  if (k > 0 && k <= kSmall) {
    // The k-th largest of the threads' maxima is at most the k-th largest logit.  Most often it is within a factor of two of the largest: then 64 counters
    // of what lies so many 2^17 units of the last place below that say where it is; else its first 16 bits, four at a time, a wave for each value of them.
    const unsigned most = ordered(top);
    unsigned cut = most;
    if (tid == 0) s.size = 0;
    if (k > 1) {
      if (tid < 64) s.count[tid] = 0;
      __syncthreads();
      const unsigned below = (most - ordered(mine)) >> 17;
      if (below < 64) atomicAdd(&s.count[below], 1u);
      __syncthreads();
      const int upto = wave_prefix((int)s.count[lane], lane);
      const u64 there = __ballot(upto >= k);
      cut = there != 0 ? most - ((unsigned)(__builtin_ctzll(there) + 1) << 17) + 1u : 0;
    }
    if (cut == 0) {
      unsigned key[kThreads / 64];
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) key[i] = ordered(s.tops[i * 64 + lane]);
#pragma unroll 1
      for (int shift = 28; shift >= 16; shift -= 4) {
        const unsigned next = cut | (unsigned)wave << shift;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) n += __builtin_popcountll(__ballot(key[i] >= next));
        unsigned* const of = s.count + 4 * shift;   // each round its own, and not the counters above
        if (lane == 0) of[wave] = (unsigned)n;
        __syncthreads();
        const u64 reach = __ballot(lane < 16 && (int)of[lane & 15] >= k);   // of 0 always
        cut |= (unsigned)(63 - __builtin_clzll(reach)) << shift;
      }
    }
    if (k == 1) __syncthreads();
    const unsigned lowest = ordered(-3.402823466e38f);
    const float least = value_of(cut > lowest ? cut : lowest);
    row.each(wave, lane, [&](u32x4 v, int t) {
      Row<T>::between(v, t, least, INFINITY, append);
    });
    __syncthreads();
    const int n = s.size;
    if (n <= kList) {
      sort(s, n, tid);
      if (wave == 0) {
        double upto = 0.0;
        last_of(n, 0, 0.0, true, k, 0.0, &upto);
        if (by_p) last_of(min(n, k), 0, 0.0, false, 0, (double)p * upto, &upto);
      }
      __syncthreads();
      const int m = s.kept;   // k at most
      // every kept entry adds up those with lower numbers
      double w = 0.0;
      if (tid < m) {
        w = weight.any(logit_of(s.list[tid]));
        w = w >= (double)q ? w : 0.0;
        s.weights[tid] = w;
      }
      __syncthreads();
      double before = 0.0;
      if (tid < m) {
        const int own = token_of(s.list[tid]);
        for (int i = 0; i < m; i += 4)
#pragma unroll
          for (int j = 0; j < 4; ++j) before += i + j < m && token_of(s.list[i + j]) < own ? s.weights[i + j] : 0.0;
      }
      __syncthreads();
      if (tid < m) s.weights[tid] = before;
      __syncthreads();
      if (wave == 0) {
        double all = 0.0;
        for (int i0 = 0; i0 < m; i0 += 64) {
          const double x = i0 + lane < m ? weight.any(logit_of(s.list[i0 + lane])) : 0.0;
          all += x >= (double)q ? x : 0.0;
        }
        all = wave_sum(all);
        // the kept entry with the highest number whose sum before it does not exceed u of them all
        const double target = share_of(all);
        int best = -1;
        float logit = 0.f;
        for (int i0 = 0; i0 < m; i0 += 64) {
          if (i0 + lane < m) {
            const u64 e = s.list[i0 + lane];
            const double x = weight.any(logit_of(e));
            if (x >= (double)q && x > 0.0 && s.weights[i0 + lane] <= target && token_of(e) > best) best = token_of(e), logit = logit_of(e);
          }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const int t = __shfl_xor(best, o, 64);
          const float x = __shfl_xor(logit, o, 64);
          if (t > best) best = t, logit = x;
        }
        if (lane == 0) finish(best, weight.any(logit), all);
      }
      return;
    }
    __syncthreads();
  }
  u64 least = 0;
  if (q > 0.f) {
    // min_p as a bound: behind the largest logit whose weight is below it.  Six bits at a time, and two; a NaN weighs nothing.
    unsigned key = 0;
    const unsigned most = ordered(top);
#pragma unroll 1
    for (int shift = 26; shift >= -4; shift -= 6) {
      const unsigned own = key | (shift >= 0 ? (unsigned)lane << shift : (unsigned)lane & 3u);
      const u64 below = __ballot(own < most && !(weight.any(value_of(own)) >= (double)q) && (shift >= 0 || lane < 4));
      const unsigned digit = (unsigned)__builtin_popcountll(below) - 1u;
      key |= shift >= 0 ? digit << shift : digit;
    }
    least = (u64)(key + 1) << 32 | 0x80000000u;   // with the highest number
  }
  if (k > 0 || by_p) {
    // Bins over the logits from the largest down, as far as weights matter beside 1 - top_p of the sum (and further for top_k): 2^fine of them an octave of the
    // weights, 32 at least (as far is 56 octaves at most).  Differences are halved: those of the largest numbers stay finite.
    const float reach = (logf((float)V) + (by_p ? fmaxf(-logf(1.f - p), 0.f) : 0.f) + 3.f) * 1.4426950408889634f;
    int fine = 5;
    while (fine < 9 && reach * (float)(2 << fine) <= (float)(kBins - 1)) ++fine;
    const float step = (float)fmin(fmax(weight.c * (double)(2 << fine), 2e-38), 3e38), half = 0.5f * top;
    const auto bin_of = [&](float x) __attribute__((always_inline)) -> int { return (int)fminf(fmaf(x, -0.5f, half) * step, (float)(kBins - 1)); };
    for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
    __syncthreads();
    // the last bin's, which may be most, add up on their way
    const auto histogram = [&](auto counted) __attribute__((always_inline)) {
      u64 far = 0;
      int far_count = 0;
      row.each(wave, lane, [&](u32x4 v, int) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float x = Row<T>::value(v, j);
          if (x > -INFINITY) {
            const int at = bin_of(x);
            const u64 w = integer(weight.any(x, at >> fine));
            if (at < kBins - 1) {
              atomicAdd(&s.mass[at], w);
              if (counted) atomicAdd(&s.count[at], 1u);
            } else {
              far += w;
              far_count += 1;
            }
          }
        }
      });
      far = wave_sum(far);
      far_count = wave_sum(far_count);
      if (lane == 0) {
        atomicAdd(&s.mass[kBins - 1], far);
        atomicAdd(&s.count[kBins - 1], (unsigned)far_count);
      }
    };
    if (k > 0) histogram(std::integral_constant<bool, true>());
    else histogram(std::integral_constant<bool, false>());   // top_p asks for no ranks
    __syncthreads();
    // The bin where the order reaches `most` entries, or a weight of `target` (below 0: top_p of them all); what lies before it.  Of the order's bins, or (octave
    // >= 0) of the parts of one in that octave.
    const auto choose = [&](bool by_rank, int most, double target, int octave) __attribute__((always_inline)) {
      if (wave == 0) {
        const auto octave_of = [&](int i) __attribute__((always_inline)) -> int { return octave >= 0 ? octave : i >> fine; };
        u64 m = 0;   // a lane's bins lie in one octave
        int n = 0;
        for (int i = 0; i < kBins / 64; ++i) m += s.mass[lane * (kBins / 64) + i], n += (int)s.count[lane * (kBins / 64) + i];
        const double um = wave_prefix(value_in(m, octave_of(lane * (kBins / 64))), lane), mb = __shfl_up(um, 1, 64);
        const int un = wave_prefix(n, lane);
        if (!by_rank && target < 0.0) {
          target = (double)p * __shfl(um, 63, 64);
          if (lane == 0) s.target = target;
        }
        // the lane whose bins reach it; the last one with entries if none does
        const bool any = by_rank ? n > 0 : m > 0, reaches = any && (by_rank ? un >= most : um >= target);
        const u64 r = __ballot(reaches), some = __ballot(any);
        const int who = r != 0 ? __builtin_ctzll(r) : 63 - __builtin_clzll(some);
        // its bins, one a lane
        const int at = __shfl(lane, who, 64) * (kBins / 64) + (lane & 31);
        const double base_m = __shfl(lane > 0 ? mb : 0.0, who, 64);
        const int base_n = __shfl(un - n, who, 64);
        const double w = lane < 32 ? value_in(s.mass[at], octave_of(at)) : 0.0;
        const int c = lane < 32 ? (int)s.count[at] : 0;
        const double upto_m = base_m + wave_prefix(w, lane), below = __shfl_up(upto_m, 1, 64);
        const int upto_n = base_n + wave_prefix(c, lane);
        const bool own = by_rank ? c > 0 : w > 0.0;
        const u64 hit = __ballot(own && (by_rank ? upto_n >= most : upto_m >= target)), full = __ballot(own);
        const int bin = hit != 0 ? __builtin_ctzll(hit) : 63 - __builtin_clzll(full);
        if (lane == bin) {
          s.before = lane > 0 ? below : base_m;
          s.ranks_before = upto_n - c;
          s.bin = at;
          s.size = 0;
        }
      }
      __syncthreads();
    };
    // All entries of a bin, sorted: from a bin of more than the list holds, the part of it where the order reaches its end.
    const auto gather = [&](bool by_rank, int most) __attribute__((always_inline)) {
      choose(by_rank, most, -1.0, -1);
      const int bin = s.bin;
      const double target = by_rank ? 0.0 : s.target;
      const float width = 1.f / step, slack = 1e-4f * width * (float)(bin + 1) + 5e-7f * fabsf(top);   // of halves, as in bin_of
      const float to = 2.f * (half - (width * (float)bin - slack)),
                  from = bin == kBins - 1 ? -3.402823466e38f : fmaxf(2.f * (half - (width * (float)(bin + 1) + slack)), -3.402823466e38f);
      // entries lo ... hi of the order are left; each pass leaves a part of 2048 of them
      u64 lo = bound, hi = ~0ull;   // nothing that top_k left out
      // the logits that the bin can hold, and a little more: what they are exactly is asked of few
      const auto in_bin = [&](u32x4 v, int t, auto other) __attribute__((always_inline)) {
        Row<T>::between(v, t, from, to, [&](float x, int tk) __attribute__((always_inline)) {
          if (x > -INFINITY) {
            const int at = bin_of(x);
            const u64 e = entry(x, tk);
            if (at < bin) other(x);
            if (at == bin && e >= lo && e <= hi) append(x, tk);
          }
        });
      };
      // on the way, the sums of the weights before the bin (and from min_p's bound on), which are kept whatever is left of the bin itself
      sum = 0.0;
      const float beyond = fmaxf(value_of(ordered(fmaxf(to, weight.floor)) + 1u), least != 0 ? logit_of(least) : -INFINITY);
      row.each(wave, lane, [&](u32x4 v, int t) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float x = Row<T>::value(v, j);
          const double w = weight(x);
          sum += x >= beyond ? w : 0.0;
          if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        in_bin(v, t, [&](float x) { sum += least == 0 || x >= logit_of(least) ? weight.any(x) : 0.0; });
      });
      __syncthreads();
      int n = s.size;
      summed = n <= kList;
      __syncthreads();
      while (n > kList) {
        // the range of what is left
        if (tid == 0) s.list[0] = ~0ull, s.list[1] = 0;
        __syncthreads();
        u64 least = ~0ull, most_e = 0;
        row.each(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
            if (x > -INFINITY && bin_of(x) == bin) {
              const u64 e = entry(x, tk);
              if (e >= lo && e <= hi) {
                least = e < least ? e : least;
                most_e = e > most_e ? e : most_e;
              }
            }
          });
        });
        atomicMin(&s.list[0], least);
        atomicMax(&s.list[1], most_e);
        for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
        __syncthreads();
        lo = s.list[0];
        hi = s.list[1];
        int shift = 0;
        while ((hi - lo) >> shift >= kBins) ++shift;
        const double before = s.before;
        const int ranks = s.ranks_before;
        __syncthreads();
        row.each(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
            if (x > -INFINITY && bin_of(x) == bin) {
              const u64 e = entry(x, tk);
              if (e >= lo && e <= hi) {
                const int at = (int)((hi - e) >> shift);
                atomicAdd(&s.mass[at], integer(weight.any(x, bin >> fine)));
                atomicAdd(&s.count[at], 1u);
              }
            }
          });
        });
        __syncthreads();
        choose(by_rank, most - ranks, target > before ? target - before : 0.0, bin >> fine);
        const int sub = s.bin;
        const u64 top_e = hi - ((u64)sub << shift);
        const u64 width = (1ull << shift) - 1;
        lo = top_e - lo > width ? top_e - width : lo;
        hi = top_e;
        if (tid == 0) s.before += before, s.ranks_before += ranks;
        __syncthreads();
        row.each(wave, lane, [&](u32x4 v, int t) __attribute__((always_inline)) { in_bin(v, t, [](float) {}); });
        __syncthreads();
        n = s.size;
        __syncthreads();
      }
      sort(s, n, tid);
      return n;
    };
    if (k > 0) {
      const int n = gather(true, k);
      if (wave == 0) {
        double upto = 0.0;
        const u64 e = last_of(n, s.ranks_before, s.before, true, k, 0.0, &upto);
        if (lane == 0) s.bound = e;
      }
      __syncthreads();
      bound = s.bound;
      __syncthreads();
      if (by_p) {   // the histogram anew: gathering may have used it, and what top_k leaves out counts no more
        for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
        __syncthreads();
        row.each(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
            if (x > -INFINITY && entry(x, tk) >= bound) {
              atomicAdd(&s.mass[bin_of(x)], integer(weight.any(x, bin_of(x) >> fine)));
              atomicAdd(&s.count[bin_of(x)], 1u);
            }
          });
        });
        __syncthreads();
      }
    }
    if (by_p) {
      const int n = gather(false, 0);
      if (wave == 0) {
        double upto = 0.0;
        const u64 e = last_of(n, s.ranks_before, s.before, false, 0, s.target, &upto);
        if (lane == 0) s.bound = e > bound ? e : bound;
      }
      __syncthreads();
      bound = s.bound;
    }
  }
  bound = bound > least ? bound : least;
  // ---------------------------------------------------------------------------
  // The draw: sums of the kept weights, of each wave's part of the row, then of a sixteenth of one part by each wave.
  // ---------------------------------------------------------------------------
  // Kept are logits from `last_logit` on, with numbers behind last_token those above it.  All of them are numbers that the weight takes.
  float last_logit = bound != 0 ? logit_of(bound) : weight.floor;
  const int last_token = bound == 0 || last_logit < weight.floor ? 0x7fffffff : token_of(bound);
  last_logit = fmaxf(last_logit, weight.floor);
  const float above = value_of(ordered(last_logit) + 1u);
  const auto sum_of = [&](u32x4 v, int t, auto each_of) __attribute__((always_inline)) {
    const float from = t > last_token ? above : last_logit;
    if (t <= last_token && t + P - 1 > last_token) {   // the one piece with numbers on both sides
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (t + j > last_token && Row<T>::value(v, j) < above) Row<T>::drop(v, j);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const float x = Row<T>::value(v, j);
      const double w = weight(x);
      each_of(x >= from ? w : 0.0, t + j);
      if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // eight polynomials at once do not fit the registers
    }
  };
  const auto add = [&](double w, int) __attribute__((always_inline)) { sum += w; };
  bool weighed = everything && !row.infinite;
  if (weighed) {
    // a wave without logits beside its first ones has none, or is weighed again, and so are all
    const bool none = !(wave_max(mine) > -INFINITY);
    const bool held = fabsf(beside) < INFINITY && ((double)top - (double)beside) * weight.c <= 900.0;
    sum = held && !none ? sum * weight.any(beside) : 0.0;
    if (!held && !none && lane == 0) s.again = 1;
    if (lane == 0) s.sums[wave] = sum;
    __syncthreads();
    weighed = s.again == 0;
    __syncthreads();
  }
  if (!weighed && summed) {
    for (int i = lane; i < s.kept; i += 64) {
      const int piece = (token_of(s.list[i]) - row.begin) / P;
      if (piece / (64 * row.pieces) == wave && s.list[i] >= bound) sum += weight.any(logit_of(s.list[i]));
    }
    sum = wave_sum(sum);
    if (lane == 0) s.sums[wave] = sum;
    __syncthreads();
    weighed = true;
  }
  if (!weighed) {
    sum = 0.0;
    row.each(wave, lane, [&](u32x4 v, int t) __attribute__((always_inline)) {
      if (Row<T>::largest(v) >= last_logit) sum_of(v, t, add);
    });
    sum = wave_sum(sum);
    if (lane == 0) s.sums[wave] = sum;
    __syncthreads();
  }
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) all += s.sums[i];
  double rest = share_of(all);
  // the part: the first behind which the sums exceed `rest`; with a random number of 1 or more the last that holds anything
  const auto locate = [&](const double* sums, double& rest) __attribute__((always_inline)) -> int {
    int part = -1;
    for (int i = 0; i < kWaves; ++i) {
      if (!(sums[i] > 0.0)) continue;
      if (part >= 0) rest -= sums[part];
      part = i;
      if (rest < sums[i]) break;
    }
    return part;
  };
  const int part = locate(s.sums, rest);
  const int each = (row.pieces + kWaves - 1) / kWaves, begin = wave * each, end = min(begin + each, row.pieces);
  sum = 0.0;
  for (int i = begin; i < end; ++i) {
    const int piece = row.piece(part, lane, i);
    sum_of(row.fetch(piece), row.begin + piece * P, add);
  }
  sum = wave_sum(sum);
  if (lane == 0) s.scan[wave] = sum;
  __syncthreads();
  const int sub = locate(s.scan, rest);
  if (wave != sub) return;
  // 64 pieces at a time: the last with a weight whose sums before it do not exceed `rest`
  int token = -1;
  double chosen = 0.0;
  for (int i = begin; i < end; ++i) {
    const int piece = row.piece(part, lane, i);
    const u32x4 v = row.fetch(piece);
    const int t = row.begin + piece * P;
    sum = 0.0;
    sum_of(v, t, add);
    const double w = sum;
    const double upto = wave_prefix(w, lane), before = upto - w;
    const u64 some = __ballot(w > 0.0), reach = __ballot(w > 0.0 && rest < upto);
    if (some == 0) continue;
    const int who = reach != 0 ? __builtin_ctzll(reach) : 63 - __builtin_clzll(some);
    int tk = -1;
    double wt = 0.0, left = rest - before;
    sum_of(v, t, [&](double x, int token_at) __attribute__((always_inline)) {
      if (x > 0.0 && (tk < 0 || left >= 0.0)) tk = token_at, wt = x;
      left -= x;
    });
    token = __shfl(tk, who, 64);
    chosen = __shfl(wt, who, 64);
    if (reach != 0) break;
    rest -= __shfl(upto, 63, 64);
  }
  if (lane == 0) finish(token, chosen, all);
}

dark_status check(const dark_sample_params* p) {
  if (p == nullptr || p->B < 0 || p->V <= 0) return DARK_EINVAL;
  if (p->io_dtype != DARK_F32 && p->io_dtype != DARK_BF16) return DARK_EINVAL;
  if (!(p->temperature >= 0.f) || std::isnan(p->top_p) || std::isnan(p->min_p)) return DARK_EINVAL;
  if (p->V > (1 << 27) || p->B > (1 << 22)) return DARK_EUNSUPPORTED;
  return DARK_OK;
}

}  // namespace
}  // namespace sample
}  // namespace dark

using namespace dark;

extern "C" {

dark_status dark_sample(const dark_sample_params* p, const void* logits, const float* uniform, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, int32_t* out_token, float* out_logprob,
                        void* hip_stream) {
  DARK_TRY(sample::check(p));
  if (p->B == 0) return DARK_OK;
  if (logits == nullptr || out_token == nullptr) return DARK_EINVAL;
  if (uniform == nullptr && (temperature != nullptr || p->temperature > 0.f)) return DARK_EINVAL;   // nothing to draw by
  if (!aligned(logits, 16) || !aligned(uniform, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
      !aligned(min_p, 4) || !aligned(out_token, 4) || !aligned(out_logprob, 4))
    return DARK_EALIGN;
  const size_t rows = 4 * (size_t)p->B, size = (size_t)p->B * p->V * (p->io_dtype == DARK_BF16 ? 2 : 4);
  if (overlap({{out_token, rows}, {out_logprob, rows}},
              {{logits, size}, {uniform, rows}, {temperature, rows}, {top_k, rows}, {top_p, rows}, {min_p, rows}}))
    return DARK_EINVAL;
  const sample::Setting set{temperature, top_p, min_p, top_k, p->temperature, p->top_p, p->min_p, p->top_k};
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const dim3 grid((unsigned)std::min(p->B, sample::kMostGroups), (unsigned)((p->B - 1) / sample::kMostGroups + 1));
#define DARK_SAMPLE(T)                                                                                                              \
  DARK_LAUNCH(KID_SAMPLE, st, (sample::k_sample<T>), grid, dim3(sample::kThreads), 0, static_cast<const T*>(logits), uniform, set, out_token, out_logprob, p->B, p->V)
  if (p->io_dtype == DARK_BF16) {
    DARK_SAMPLE(unsigned short);
  } else {
    DARK_SAMPLE(float);
  }
#undef DARK_SAMPLE
  return DARK_OK;
}

}  // extern "C"
