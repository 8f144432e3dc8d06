// Drawing the next token of every row from its logits: temperature, top_k, top_p, min_p, by a given random number.
//
// With w_t = exp((x_t - max x) / T) and the tokens in order of their logits (equal ones by their number), a row keeps the first top_k of them; of
// those, the shortest beginning that holds top_p of their sum; and of those the ones with w_t >= min_p.  The token drawn is the first, in
// the order of the tokens' numbers, behind which the kept weights add up to more than u times their sum.
//
// A workgroup takes a row.  What is kept but for min_p is a beginning of the order, so that two numbers say it: the last kept logit, and the last
// kept token of that logit.  Small top_k: a bound from the threads' maxima leaves few candidates, which are sorted in LDS.  Else
// a histogram of weights (in integers, whose sums have no order) over the logits finds the bin where the beginning ends, and the bin's
// entries are sorted.  The draw sums the kept weights by waves, each of which holds a contiguous part of the row, and looks into one of them.
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
constexpr float kLog2e = 1.4426950408889634f;

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
  int begin, V, pieces;   // token of the row's first piece's first element (it may lie before the row); tokens; pieces of a wave, in 64s
  bool held;
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
    held = pieces <= kHeld;
    if (held) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) r[i] = i < pieces ? fetch(piece(wave, lane, i)) : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
    }
  }
  __device__ static float value(u32x4 v, int j) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(j & 1 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16);
    else return __uint_as_float(v[j]);
  }
  // the same without the held ones, for what is rarely needed: less code
  template <typename F>
  __device__ void again(int wave, int lane, const F& f) const {
#pragma unroll 1
    for (int i = 0; i < pieces; ++i) f(fetch(piece(wave, lane, i)), begin + piece(wave, lane, i) * P);
  }
  // f(piece, its first token) for the thread's pieces
  template <typename F>
  __device__ void each(int wave, int lane, const F& f) const {
    if (held) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i < pieces) f(r[i], begin + piece(wave, lane, i) * P);
    } else {
#pragma unroll 2
      for (int i = 0; i < pieces; ++i) f(fetch(piece(wave, lane, i)), begin + piece(wave, lane, i) * P);
    }
  }
};

// exp((x - m) / T): the exponent (x - m) c, c = log2 e / T in two floats, keeps what its rounding leaves.
struct Weight {
  float m, c, c2;
  bool infinite;   // the largest logit is infinite: those that are share everything
  __device__ float operator()(float x) const {
    if (infinite) return x == INFINITY ? 1.f : 0.f;
    const float d = x - m, e = d * c, more = fmaf(d, c, -e) + d * c2, w = __builtin_amdgcn_exp2f(e);
    return e >= -125.f ? fmaf(w, more * 0.69314718f, w) : 0.f;   // also where x is NaN or -infinity
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
  u64 list[kList];
  u64 mass[kBins];
  unsigned count[kBins];
  double sums[kWaves];
  double scan[kWaves];
  float tops[kThreads];
  u64 bound;         // the last entry that is kept
  u64 before;        // weight of the bins before the chosen one
  int ranks_before, bin, size;
  unsigned lo, hi;
  double total;
};

// The first n entries of the list in descending order; the others are 0.
__device__ __forceinline__ void sort(Shared& s, int n, int tid) {
  int size = 64;
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
    const long long all = (first + V - base + P - 1) / P;
    row.pieces = (int)((all + kThreads - 1) / kThreads);
  }
  row.load(wave, lane);
  // the largest logit, of every thread and of all
  float mine = -INFINITY;
  row.each(wave, lane, [&](u32x4 v, int) {
#pragma unroll
    for (int j = 0; j < P; ++j) mine = fmaxf(mine, Row<T>::value(v, j));   // of a NaN and a number: the number
  });
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
  const bool greedy = !(temp > 0.f);
  int k = set.top_k != nullptr ? set.top_k[b] : set.k;
  float p = set.top_p != nullptr ? set.top_p[b] : set.p, q = set.min_p != nullptr ? set.min_p[b] : set.q, u = uniform != nullptr ? uniform[b] : 0.f;
  Weight weight;
  weight.m = top;
  weight.infinite = top == INFINITY;
  {
    const double c = greedy ? 1.0 : 1.4426950408889634 / (double)temp;
    weight.c = (float)fmin(c, 3e38);
    weight.c2 = c < 3e38 ? (float)(c - (double)weight.c) : 0.f;
  }
  if (greedy) k = 1, p = 1.f, q = 0.f;
  q = q > 0.f ? fminf(q, 1.f) : 0.f;
  if (k <= 0 || k >= V) k = 0;
  const bool by_p = p < 1.f;
  if (!(p > 0.f)) p = by_p ? 0.f : 1.f;
  u64 bound = 0;   // entries from this one on are kept
  const float high = (float)(1u << (__builtin_clz((unsigned)V) - 2));   // 2^-32 of a weight's unit: V of them stay below 2^62
  const auto integer = [&](float w) -> u64 {   // w unit, in two halves
    const float a = w * high;
    const unsigned h = (unsigned)a;
    return (u64)h << 32 | (unsigned)((a - (float)h) * 4294967296.f);
  };

  // The list holds all entries of a part of the order, sorted, behind `rank` entries of weight `held`: the last that is kept of them, by rank
  // (k > 0) or by weight (target), and the weight up to it.  By one wave.
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
      }
      sum = __shfl(up, 63, 64);
    }
    return found;
  };
  const auto append = [&](float x, int t) {
    const int at = atomicAdd(&s.size, 1);
    if (at < kList) s.list[at] = entry(x, t);
  };

  bool done = k == 0 && !by_p;
  if (!done && k > 0 && k <= kSmall) {
    // The k-th largest of the threads' maxima is at most the k-th largest logit: bisection over the 32 bits of its order, by one wave.
    if (wave == 0) {
      unsigned key[kThreads / 64], cut = 0;
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) key[i] = ordered(s.tops[i * 64 + lane]);
      for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 8); --bit) {
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
    row.each(wave, lane, [&](u32x4 v, int t) {
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (Row<T>::value(v, j) >= least) append(Row<T>::value(v, j), t + j);
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
      bound = s.bound;
      done = true;
    }
    __syncthreads();
  }
  if (!done) {
    // Bins over the logits from the largest down, as far as weights matter beside 1 - top_p of the sum (and further for top_k).
    const float reach = (logf((float)V) + (by_p ? fmaxf(-logf(1.f - p), 0.f) : 0.f) + 3.f) * 1.4426950408889634f / fmaxf(weight.c, 1e-30f);
    const float step = fminf((float)(kBins - 1) / reach, 1e30f);
    const auto bin_of = [&](float x) -> int { return weight.infinite ? (x == INFINITY ? 0 : kBins - 1) : (int)fminf((weight.m - x) * step, (float)(kBins - 1)); };
    for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
    __syncthreads();
    row.each(wave, lane, [&](u32x4 v, int) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float x = Row<T>::value(v, j);
        if (x > -INFINITY) {
          const int at = bin_of(x);
          atomicAdd(&s.mass[at], integer(weight(x)));
          atomicAdd(&s.count[at], 1u);
        }
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
        row.again(wave, lane, [&](u32x4 v, int t) {
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const float x = Row<T>::value(v, j);
            if (x > -INFINITY && bin_of(x) == bin) {
              const u64 e = entry(x, t + j);
              if (e >= lo && e <= hi) {
                least = e < least ? e : least;
                most_e = e > most_e ? e : most_e;
              }
            }
          }
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
        row.again(wave, lane, [&](u32x4 v, int t) {
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const float x = Row<T>::value(v, j);
            if (x > -INFINITY && bin_of(x) == bin) {
              const u64 e = entry(x, t + j);
              if (e >= lo && e <= hi) {
                const int at = (int)((hi - e) >> shift);
                atomicAdd(&s.mass[at], integer(weight(x)));
                atomicAdd(&s.count[at], 1u);
              }
            }
          }
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
      row.each(wave, lane, [&](u32x4 v, int t) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float x = Row<T>::value(v, j);
          if (x > -INFINITY && bin_of(x) == bin) {
            const u64 e = entry(x, t + j);
            if (e >= lo && e <= hi) append(x, t + j);
          }
        }
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
        row.again(wave, lane, [&](u32x4 v, int t) {
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const float x = Row<T>::value(v, j);
            if (x > -INFINITY && entry(x, t + j) >= bound) {
              atomicAdd(&s.mass[bin_of(x)], integer(weight(x)));
              atomicAdd(&s.count[bin_of(x)], 1u);
            }
          }
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
  const auto kept = [&](float x, int t) -> float {
    const float w = weight(x);
    return x > -INFINITY && w >= q && (bound == 0 || entry(x, t) >= bound) ? w : 0.f;
  };
  const auto sum_of = [&](u32x4 v, int t) -> float {
    float w = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) w += kept(Row<T>::value(v, j), t + j);
    return w;
  };
  double sum = 0.0;
  row.each(wave, lane, [&](u32x4 v, int t) { sum += (double)sum_of(v, t); });
  sum = wave_sum(sum);
  if (lane == 0) s.sums[wave] = sum;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) all += s.sums[i];
  const float uu = u > 0.f ? u : 0.f;
  double rest = (greedy ? 0.0 : (double)uu) * all;
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
    sum += (double)sum_of(row.fetch(piece), row.begin + piece * P);
  }
  sum = wave_sum(sum);
  if (lane == 0) s.scan[wave] = sum;
  __syncthreads();
  const int sub = locate(s.scan, rest);
  if (wave != sub) return;
  // 64 pieces at a time: the last with a weight whose sums before it do not exceed `rest`
  int token = -1;
  float chosen = 0.f;
  for (int i = begin; i < end; ++i) {
    const int piece = row.piece(part, lane, i);
    const u32x4 v = row.fetch(piece);
    const int t = row.begin + piece * P;
    const double w = (double)sum_of(v, t);
    const double upto = wave_prefix(w, lane), before = upto - w;
    const u64 some = __ballot(w > 0.0), reach = __ballot(w > 0.0 && rest < upto);
    if (some == 0) continue;
    const int who = reach != 0 ? __builtin_ctzll(reach) : 63 - __builtin_clzll(some);
    int tk = -1;
    float wt = 0.f;
    double left = rest - before;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const float x = kept(Row<T>::value(v, j), t + j);
      if (x > 0.f && (tk < 0 || left >= 0.0)) tk = t + j, wt = x;
      left -= (double)x;
    }
    token = __shfl(tk, who, 64);
    chosen = __shfl(wt, who, 64);
    if (reach != 0) break;
    rest -= __shfl(upto, 63, 64);
  }
  if (lane == 0) {
    out_token[b] = token;
    if (out_logprob != nullptr) out_logprob[b] = greedy ? 0.f : (float)log((double)chosen / all);
  }
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
  if (p->io_dtype == DARK_BF16) {
    DARK_LAUNCH(KID_SAMPLE, st, sample::k_sample<unsigned short>, dim3(p->B), dim3(sample::kThreads), 0, static_cast<const unsigned short*>(logits),
                uniform, set, out_token, out_logprob, p->V);
  } else {
    DARK_LAUNCH(KID_SAMPLE, st, sample::k_sample<float>, dim3(p->B), dim3(sample::kThreads), 0, static_cast<const float*>(logits), uniform,
                set, out_token, out_logprob, p->V);
  }
  return DARK_OK;
}

}  // extern "C"
