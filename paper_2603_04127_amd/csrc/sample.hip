// Drawing the next token of every row from its logits: temperature, top_k, top_p, min_p, by a given random number.
//
// With w_t = exp((x_t - max x) / T) and the tokens in order of their logits (equal ones by their number), a row keeps the first top_k of them; of
// those, the shortest beginning that holds top_p of their sum; and of those the ones with w_t >= min_p.  The token drawn is the first, in
// the order of the tokens' numbers, behind which the kept weights add up to more than u times their sum.
//
// A workgroup takes a row, whose 16-byte pieces its threads hold where they have room for them.  What is kept but for min_p is a beginning of the
// order, so that its last entry says it.  Small top_k: a bound from the threads' maxima leaves few candidates, which count those before them
// and, kept, the weights of those with lower numbers: no further pass.  Else a histogram of weights over the logits finds the bin
// where the beginning ends, and the bin's entries are sorted.  The draw sums the kept weights by waves, each of which holds a
// contiguous part of the row, and looks into one of them.
// Weights are in fp64, by a polynomial, to 2^-31 of their value, and so are their sums; a histogram's are integers, whose sums have no order.
// In fp32 the borders between a large row's tokens would be off by some 2^-30 of the row's sum each, 2^17 of them together by 2^-13: one
// row in 8000 would draw a token's neighbour.
#include <cmath>

#include "common.h"

namespace dark {
namespace sample {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kHeld = 16;      // pieces of 16 bytes that a thread holds; longer rows are read anew in every pass
constexpr int kBins = 2048;
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
  u32x4 r[kHeld];
  __device__ u32x4 fetch(int piece) const {   // -infinity where there is no token
    u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(at, (unsigned)piece * 16u, 0, 0);
    const int t = begin + piece * P;
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
    return v;
  }
  __device__ int piece(int wave, int lane, int i) const { return (wave * pieces + i) * 64 + lane; }
  __device__ void load(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < pieces) r[i] = fetch(piece(wave, lane, i));
  }
  __device__ static float value(u32x4 v, int j) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(j & 1 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16);
    else return __uint_as_float(v[j]);
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
  // f(piece, its first token) for the thread's pieces
  template <bool HELD, typename F>
  __device__ __forceinline__ void each(int wave, int lane, const F& f) const {
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i < pieces) f(r[i], begin + piece(wave, lane, i) * P);
    } else {
#pragma unroll 1
      for (int i = 0; i < pieces; ++i) f(fetch(piece(wave, lane, i)), begin + piece(wave, lane, i) * P);
    }
  }
};

// exp((x - m) / T) = 2^z: the sum of z^k ln 2^k / k! up to k = 8 for what rounding z leaves, at most 1/2: off by 2^-32.
struct Weight {
  double m, c;     // c = log2 e / T
  float top;
  bool infinite;   // the largest logit is infinite: those that are share everything
  __device__ __forceinline__ double operator()(float x) const {
    const double z = infinite ? (x == INFINITY ? 0.0 : -2000.0) : ((double)x - m) * c, n = rint(z), f = z - n;
    double y = fma(f, 1.3215486790144309e-6, 1.5252733804059841e-5);
    y = fma(f, y, 1.5403530393381609e-4);
    y = fma(f, y, 1.3333558146428443e-3);
    y = fma(f, y, 9.6181291076284772e-3);
    y = fma(f, y, 5.5504108664821580e-2);
    y = fma(f, y, 2.4022650695910071e-1);
    y = fma(f, y, 6.9314718055994531e-1);
    y = fma(f, y, 1.0);
    return z > -1000.0 ? ldexp(y, (int)n) : 0.0;   // also where x is NaN or -infinity
  }
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
  u64 list[kList], sorted[kCounted];
  u64 mass[kBins];
  unsigned count[kBins];
  double sums[kWaves], scan[kWaves], weights[kSmall];
  float tops[kThreads];
  u64 bound;         // the last entry that is kept
  u64 before;        // weight of the bins before the chosen one
  int ranks_before, bin, size, kept;
  unsigned lo;
};

// The list's first n entries in descending order.
__device__ __forceinline__ void sort(Shared& s, int n, int tid) {
  if (n <= kCounted) {
    const u64 own = tid < n ? s.list[tid] : 0;
    int before = 0;
    if (tid < n)
#pragma unroll 4
      for (int i = 0; i < n; ++i) before += s.list[i] > own;
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

template <typename T, bool HELD>
__global__ __launch_bounds__(kThreads) void k_sample(const T* __restrict__ logits, const float* __restrict__ uniform, Setting set,
                                                     int32_t* __restrict__ out_token, float* __restrict__ out_logprob, int V) {
  __shared__ Shared s;
  // Bit 9 of MODE, IEEE, off: a maximum of a signalling NaN and a number is the number.
  __builtin_amdgcn_s_setreg(1 | 9 << 6, 0);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
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
  if (HELD) row.load(wave, lane);
  // the largest logit, of every thread and of all
  float mine = -INFINITY;
  row.template each<HELD>(wave, lane, [&](u32x4 v, int) { mine = fmaxf(mine, Row<T>::largest(v)); });   // of a NaN and a number: the number
  s.tops[tid] = mine;
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
  const float temp = set.temperature != nullptr ? set.temperature[b] : set.T;
  int k = set.top_k != nullptr ? set.top_k[b] : set.k;
  float p = set.top_p != nullptr ? set.top_p[b] : set.p, q = set.min_p != nullptr ? set.min_p[b] : set.q, u = uniform != nullptr ? uniform[b] : 0.f;
  Weight weight;
  weight.m = top;
  weight.infinite = top == INFINITY;
  weight.c = fmin(1.4426950408889634 / (double)temp, 1e300);
  if (!(temp > 0.f)) {   // the largest logit
    weight.c = 1.0;
    k = 1;
    p = 1.f;
  }
  q = q > 0.f ? fminf(q, 1.f) : 0.f;
  u = u > 0.f ? u : 0.f;
  if (k <= 0 || k >= V) k = 0;
  const bool by_p = p < 1.f;
  if (!(p > 0.f)) p = by_p ? 0.f : 1.f;
  u64 bound = 0;   // entries from this one on are kept
  const double unit = (double)(1ull << (__builtin_clz((unsigned)V) + 19));   // of an integer weight: V of them stay below 2^51
  const auto integer = [&](double w) -> u64 { return (u64)__double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull; };

  // The list holds all entries of a part of the order, sorted, behind `rank` entries of weight `held`: the last that is kept of them, by rank
  // or by weight (target), and the weight up to it.  By one wave.
  const auto last_of = [&](int n, int rank, u64 held, bool by_rank, int most, u64 target, u64* upto) -> u64 {
    u64 found = 0, sum = held;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const u64 e = i0 + lane < n ? s.list[i0 + lane] : 0;
      const u64 w = e != 0 ? integer(weight(logit_of(e))) : 0;
      const u64 up = sum + wave_prefix(w, lane);
      const bool in = e != 0 && (by_rank ? rank + i0 + lane < most : up - w < target || rank + i0 + lane == 0);
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
  const auto append = [&](float x, int t) {
    const int at = atomicAdd(&s.size, 1);
    if (at < kList) s.list[at] = entry(x, t);
  };
  const auto finish = [&](int token, double w, double all) {
    out_token[b] = token;
    if (out_logprob != nullptr) out_logprob[b] = (float)log(w / all);
  };

  bool done = k == 0 && !by_p;
  if (!done && k > 0 && k <= kSmall) {
    // The k-th largest of the threads' maxima is at most the k-th largest logit: its first bits, by one wave.
    if (wave == 0) {
      unsigned key[kThreads / 64], cut = 0;
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) key[i] = ordered(s.tops[i * 64 + lane]);
      for (int bit = 31; bit >= 16; --bit) {
        const unsigned next = cut | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) n += __builtin_popcountll(__ballot(key[i] >= next));
        if (n >= k) cut = next;
      }
      const unsigned least = ordered(-3.402823466e38f);
      if (lane == 0) s.lo = cut > least ? cut : least, s.size = 0;
    }
    __syncthreads();
    const float least = value_of(s.lo);
    row.template each<HELD>(wave, lane, [&](u32x4 v, int t) {
      if (Row<T>::largest(v) >= least)
        Row<T>::elements(v, t, [&](float x, int tk) {
          if (x >= least) append(x, tk);
        });
    });
    __syncthreads();
    const int n = s.size;
    if (n <= kList) {
      sort(s, n, tid);
      if (wave == 0) {
        u64 upto = 0, e = last_of(n, 0, 0, true, k, 0, &upto);
        if (by_p) e = last_of(min(n, k), 0, 0, false, 0, (u64)((double)p * (double)upto), &upto);
        if (lane == 0) s.bound = e;
      }
      __syncthreads();
      const int m = s.kept;
      if (m <= kSmall) {
        // every kept entry adds up those with lower numbers
        double w = 0.0;
        if (tid < m) {
          w = weight(logit_of(s.list[tid]));
          w = w >= (double)q ? w : 0.0;
          s.weights[tid] = w;
        }
        __syncthreads();
        double before = 0.0;
        if (tid < m) {
          const int own = token_of(s.list[tid]);
          for (int i = 0; i < m; ++i) before += token_of(s.list[i]) < own ? s.weights[i] : 0.0;
        }
        __syncthreads();
        if (tid < m) s.weights[tid] = before;
        __syncthreads();
        if (wave == 0) {
          double all = 0.0;
          for (int i0 = 0; i0 < m; i0 += 64) {
            const double x = i0 + lane < m ? weight(logit_of(s.list[i0 + lane])) : 0.0;
            all += x >= (double)q ? x : 0.0;
          }
          all = wave_sum(all);
          // the kept entry with the highest number whose sum before it does not exceed u of them all
          const double target = (double)u * all;
          int best = -1;
          float logit = 0.f;
          for (int i0 = 0; i0 < m; i0 += 64) {
            if (i0 + lane < m) {
              const u64 e = s.list[i0 + lane];
              const double x = weight(logit_of(e));
              if (x >= (double)q && x > 0.0 && s.weights[i0 + lane] <= target && token_of(e) > best) best = token_of(e), logit = logit_of(e);
            }
          }
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) {
            const int t = __shfl_xor(best, o, 64);
            const float x = __shfl_xor(logit, o, 64);
            if (t > best) best = t, logit = x;
          }
          if (lane == 0) finish(best, weight(logit), all);
        }
        return;
      }
      bound = s.bound;
      done = true;
    }
    __syncthreads();
  }
  if (!done) {
    // Bins over the logits from the largest down, as far as weights matter beside 1 - top_p of the sum (and further for top_k).
    const float reach = (logf((float)V) + (by_p ? fmaxf(-logf(1.f - p), 0.f) : 0.f) + 3.f) * 1.4426950408889634f / (float)fmin(fmax(weight.c, 1e-30), 1e30);
    const float step = fminf((float)(kBins - 1) / reach, 1e30f);
    const auto bin_of = [&](float x) -> int { return weight.infinite ? (x == INFINITY ? 0 : kBins - 1) : (int)fminf((top - x) * step, (float)(kBins - 1)); };
    for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
    __syncthreads();
    row.template each<HELD>(wave, lane, [&](u32x4 v, int) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float x = Row<T>::value(v, j);
        if (x > -INFINITY) {
          const int at = bin_of(x);
          atomicAdd(&s.mass[at], integer(weight(x)));
          atomicAdd(&s.count[at], 1u);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __syncthreads();
    // The bin where the order reaches `most` entries, or a weight of `target`; what lies before it.
    const auto choose = [&](bool by_rank, int most, u64 target) {
      if (wave == 0) {
        u64 m = 0;
        int n = 0;
        for (int i = 0; i < kBins / 64; ++i) m += s.mass[lane * (kBins / 64) + i], n += (int)s.count[lane * (kBins / 64) + i];
        u64 mb = wave_prefix(m, lane) - m;
        int nb = wave_prefix(n, lane) - n;
        // the lane whose bins reach it; the last one with entries if none does
        const bool reaches = n > 0 && (by_rank ? nb + n >= most : mb + m >= target);
        const u64 r = __ballot(reaches), some = __ballot(n > 0);
        const int who = r != 0 ? __builtin_ctzll(r) : 63 - __builtin_clzll(some);
        if (lane == who) {
          int bin = -1;
          for (int i = 0; i < kBins / 64; ++i) {
            const int c = (int)s.count[lane * (kBins / 64) + i];
            const u64 w = s.mass[lane * (kBins / 64) + i];
            if (c == 0) continue;
            if (bin >= 0) {
              if (by_rank ? nb >= most : mb >= target) break;   // reached before this one
            }
            bin = lane * (kBins / 64) + i;
            s.before = mb;
            s.ranks_before = nb;
            mb += w;
            nb += c;
          }
          s.bin = bin;
          s.size = 0;
        }
      }
      __syncthreads();
    };
    // All entries of a bin, sorted: from a bin of more than the list holds, the part of it where the order reaches its end.
    const auto gather = [&](bool by_rank, int most, u64 target) {
      choose(by_rank, most, target);
      const int bin = s.bin;
      // entries lo ... hi of the order are left; each pass leaves a part of 2048 of them
      u64 lo = bound, hi = ~0ull;   // nothing that top_k left out
      int n = (int)s.count[bin];
      __syncthreads();
      while (n > kList) {
        // the range of what is left
        if (tid == 0) s.list[0] = ~0ull, s.list[1] = 0;
        __syncthreads();
        u64 least = ~0ull, most_e = 0;
        row.template each<false>(wave, lane, [&](u32x4 v, int t) {
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
        const u64 before = s.before;
        const int ranks = s.ranks_before;
        __syncthreads();
        row.template each<false>(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
            if (x > -INFINITY && bin_of(x) == bin) {
              const u64 e = entry(x, tk);
              if (e >= lo && e <= hi) {
                const int at = (int)((hi - e) >> shift);
                atomicAdd(&s.mass[at], integer(weight(x)));
                atomicAdd(&s.count[at], 1u);
              }
            }
          });
        });
        __syncthreads();
        choose(by_rank, most - ranks, target > before ? target - before : 0);
        const int sub = s.bin;
        n = (int)s.count[sub];
        const u64 top_e = hi - ((u64)sub << shift);
        const u64 width = (1ull << shift) - 1;
        lo = top_e - lo > width ? top_e - width : lo;
        hi = top_e;
        if (tid == 0) s.before += before, s.ranks_before += ranks;
        __syncthreads();
      }
      row.template each<HELD>(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
          if (x > -INFINITY && bin_of(x) == bin) {
            const u64 e = entry(x, tk);
            if (e >= lo && e <= hi) append(x, tk);
          }
        });
      });
      __syncthreads();
      sort(s, n, tid);
      return n;
    };
    u64 whole = 0;
    for (int i = 0; i < kBins; i += 64) whole += s.mass[i + lane];
    whole = wave_sum(whole);
    __syncthreads();
    if (k > 0) {
      const int n = gather(true, k, 0);
      if (wave == 0) {
        u64 upto = 0;
        const u64 e = last_of(n, s.ranks_before, s.before, true, k, 0, &upto);
        if (lane == 0) s.bound = e, s.before = upto;
      }
      __syncthreads();
      bound = s.bound;
      whole = s.before;
      __syncthreads();
      if (by_p) {   // the histogram anew: gathering may have used it, and what top_k leaves out counts no more
        for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
        __syncthreads();
        row.template each<false>(wave, lane, [&](u32x4 v, int t) {
          Row<T>::elements(v, t, [&](float x, int tk) {
            if (x > -INFINITY && entry(x, tk) >= bound) {
              atomicAdd(&s.mass[bin_of(x)], integer(weight(x)));
              atomicAdd(&s.count[bin_of(x)], 1u);
            }
          });
        });
        __syncthreads();
      }
    }
    if (by_p) {
      const u64 target = (u64)((double)p * (double)whole);
      const int n = gather(false, 0, target);
      if (wave == 0) {
        u64 upto = 0;
        const u64 e = last_of(n, s.ranks_before, s.before, false, 0, target, &upto);
        if (lane == 0) s.bound = e > bound ? e : bound;
      }
      __syncthreads();
      bound = s.bound;
    }
  }
  // ---------------------------------------------------------------------------
  // The draw: sums of the kept weights, of each wave's part of the row, then of a sixteenth of one part by each wave.
  // ---------------------------------------------------------------------------
  const float last_logit = bound != 0 ? logit_of(bound) : -3.402823466e38f;
  const int last_token = bound != 0 ? token_of(bound) : 0x7fffffff;
  const auto kept = [&](float x, int t) -> double {
    const double w = weight(x);
    return (x > last_logit || (x == last_logit && t <= last_token)) && w >= (double)q ? w : 0.0;
  };
  const auto sum_of = [&](u32x4 v, int t) -> double {
    double w = 0.0;
    if (Row<T>::largest(v) >= last_logit) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        w += kept(Row<T>::value(v, j), t + j);
        __builtin_amdgcn_sched_barrier(0);   // one after the other: eight polynomials at once do not fit the registers, and four waves a SIMD wait for none
      }
    }
    return w;
  };
  double sum = 0.0;
  row.template each<HELD>(wave, lane, [&](u32x4 v, int t) { sum += sum_of(v, t); });
  sum = wave_sum(sum);
  if (lane == 0) s.sums[wave] = sum;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) all += s.sums[i];
  double rest = (double)u * all;
  // the part: the first behind which the sums exceed `rest`; with a random number of 1 or more the last that holds anything
  const auto locate = [&](const double* sums, double& rest) -> int {
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
    sum += sum_of(row.fetch(piece), row.begin + piece * P);
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
    const double w = sum_of(v, t);
    const double upto = wave_prefix(w, lane), before = upto - w;
    const u64 some = __ballot(w > 0.0), reach = __ballot(w > 0.0 && rest < upto);
    if (some == 0) continue;
    const int who = reach != 0 ? __builtin_ctzll(reach) : 63 - __builtin_clzll(some);
    int tk = -1;
    double wt = 0.0, left = rest - before;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const double x = kept(Row<T>::value(v, j), t + j);
      if (x > 0.0 && (tk < 0 || left >= 0.0)) tk = t + j, wt = x;
      left -= x;
    }
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
  // whether a thread holds its pieces (a row may begin up to a piece before its first element)
  const bool held = false && ((long long)p->V * (p->io_dtype == DARK_BF16 ? 2 : 4) + 32) / 16 <= (long long)sample::kThreads * sample::kHeld;
#define DARK_SAMPLE(T)                                                                                                              \
  if (held) DARK_LAUNCH(KID_SAMPLE, st, (sample::k_sample<T, true>), dim3(p->B), dim3(sample::kThreads), 0, static_cast<const T*>(logits), uniform, set, out_token, out_logprob, p->V); \
  else DARK_LAUNCH(KID_SAMPLE, st, (sample::k_sample<T, false>), dim3(p->B), dim3(sample::kThreads), 0, static_cast<const T*>(logits), uniform, set, out_token, out_logprob, p->V)
  if (p->io_dtype == DARK_BF16) {
    DARK_SAMPLE(unsigned short);
  } else {
    DARK_SAMPLE(float);
  }
#undef DARK_SAMPLE
  return DARK_OK;
}

}  // extern "C"
