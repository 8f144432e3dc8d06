// Beam search over recurrent states: the selection of the next beams from their logits, and the reordering of the states that
// belong to them.
//
// Selection, per batch entry with n beams: candidate (j, t) is worth score_j + logit_jt - log sum_u exp logit_ju; the n largest win,
// equal ones by the lowest j, then the lowest t.  k_beam_rows reads every logit once: a workgroup takes a slice of a row and leaves
// the slice's maximum, its sum of exponentials and its n largest logits in order.  k_beam_pick joins the sums of a batch entry's
// rows and takes the best of the sorted lists.
// Two candidates of different beams may lie closer together than fp32 resolves beside a score: offsets and comparisons are in fp64, and
// what tells them apart is then the sums.  A sum of exponentials is within 2^-19 of its value: 5 + 6 + 2 additions one after the other (a
// thread's 32 terms, the lanes, the waves; beside a NaN one more) are off by at most 14 2^-24, an exponential by 2^-23, and where the terms
// that matter lie x below the maximum, x < 19 since there are less than 2^27 of them, ln 2 2^-20 for the rounding of the exponent x log2 e < 2^5
// and 19 2^-26 for that of log2 e.
// Where fp64 resolves no more either (a score of -10^20, logits that differ by 10^-20) the logits themselves decide within a beam.
#include <cmath>

#include "common.h"

namespace dark {
namespace beam {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

struct Entry {
  float logit;
  int token;
};
struct Part {
  float top, sum;
};

// Monotone in the value for everything but NaN, which the callers replace; 0 is below every value.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// The same for doubles that are numbers or -infinity.
__device__ __forceinline__ u64 ordered64(double v) {
  const u64 u = (u64)__double_as_longlong(v);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double value64(u64 k) { return __longlong_as_double((long long)(k >> 63 ? k ^ 0x8000000000000000ull : ~k)); }

// Largest key of the wave.
template <int CTRL>
__device__ __forceinline__ unsigned dpp_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
  return o > v ? o : v;
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  v = dpp_max<0x121>(v);   // rotations within a row of 16 lanes by 1, 2, 4, 8
  v = dpp_max<0x122>(v);
  v = dpp_max<0x124>(v);
  v = dpp_max<0x128>(v);
  const unsigned a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16), c = __builtin_amdgcn_readlane(v, 32),
                 d = __builtin_amdgcn_readlane(v, 48);
  const unsigned ab = a > b ? a : b, cd = c > d ? c : d;
  return ab > cd ? ab : cd;
}

// A score that is no number, or infinite, leaves its beam without candidates: whatever is compared below is a number or -infinity.
__device__ __forceinline__ bool finite(float v) { return v > -INFINITY && v < INFINITY; }

constexpr int kMostBeams = 32;
constexpr float kLog2e = 1.4426950408889634f;

// A maximum m so large that the rounding of c = m L (below) would be more than an eighth of an exponent, or c infinite (a row masked
// by the type's lowest value): exponents are (v - m) L instead, two roundings and an instruction more.
__device__ __forceinline__ bool large(float m) { return fabsf(m) > 1048576.f; }
// c of a sum of 2^(v L - c)
__device__ __forceinline__ double origin(float m) { return large(m) ? (double)m * (double)kLog2e : (double)(m * kLog2e); }

// The first `count` lanes of a wave hold a candidate each: every one counts those before it (larger, or equal with a lower token) and
// takes that place in the list if it is one of the n.  Token -1 behind the last.
__device__ __forceinline__ void place(unsigned key, int token, int count, Entry* list, int n, int lane) {
  const u64 own = (u64)key << 32 | (unsigned)~token;
  int before = 0;
  for (int i = 0; i < count; ++i) {
    const u64 other = (u64)__builtin_amdgcn_readlane(key, i) << 32 | (unsigned)~__builtin_amdgcn_readlane(token, i);
    before += other > own;
  }
  if (lane < count && before < n) list[before] = Entry{value_of(key), token};
  if (lane == 0 && count < n) list[count] = Entry{0.f, -1};
}

// The n-th largest of the lanes' values.
__device__ __forceinline__ unsigned nth_of_lanes(unsigned v, int n, int lane) {
  unsigned w = 0;
  for (int i = 0; i < n; ++i) {
    w = wave_max(v);
    if (lane == __builtin_ctzll(__ballot(v == w))) v = 0;
  }
  return w;
}

// f(FIRST) + ... + f(FIRST + COUNT - 1) by halves: log2 COUNT roundings one after the other, and none where all terms are equal.
template <int FIRST, int COUNT, typename F>
__device__ __forceinline__ float tree(const F& f) {
  if constexpr (COUNT == 1) return f(FIRST);
  else return tree<FIRST, COUNT / 2>(f) + tree<FIRST + COUNT / 2, COUNT - COUNT / 2>(f);
}

// The element of row-relative index t, as a number that may win: NaN where there is none.
template <typename T>
__device__ __forceinline__ float number(const T* row, long long t, int V) {
  if (t < 0 || t >= V) return NAN;
  if constexpr (sizeof(T) == 2) return __uint_as_float((unsigned)row[t] << 16);
  else return row[t];
}

// A slice is 8192 elements of a row; thread t holds pieces t, t + 256, ... of 16 bytes.  Rows begin where they begin: the slices
// count from the 16-byte boundary at or before the row's first element.  Elements that are not the row's are -infinity, which like a NaN
// among the logits loses every comparison: lists hold what is larger than -infinity.
// The slice's n largest: the n-th largest of 64 groups' maxima (a lane of each of the four waves) bounds them from below, so that a
// comparison each is all that most elements cost; the few that pass are collected and each counts those before it.  Where more than 64
// pass (many equal ones, or the largest in few lanes) they are looked for one after the other in memory.
// Vector instructions bound it for bf16, memory for fp32.  Hence: 16-bit elements stay packed, and in two passes of three the upper one
// of a pair is taken with the lower one's bits behind it, which no comparison between such numbers minds; a NaN costs the sum a
// second pass instead of every element an instruction.
// (32 x 8 rows of 131,071, n = 8: 70 us when every wave took its largest out one by one, 25 with a list for every wave, 19.5 now; fp32 25.6,
// 134 MB at 5.2 TB/s.
// Slices of 2048: as many lists more for k_beam_pick; 1 x 4 rows of 32,000 4.1 + 6.2 us against 4.6 + 5.4, 1 x 8 of 131,071 4.7 + 10.9
// against 5.8 + 6.7, 16 x 8 of them 19 + 12 against 12.4 + 7.3.  Of 16,384: no faster, and more registers for fp32.)
constexpr int kMostPassed = 64, kEach = 32, kSlice = 256 * kEach;
template <typename T>
__global__ __launch_bounds__(256, 8) void k_beam_rows(const T* __restrict__ logits, const float* __restrict__ scores,
                                                      const unsigned char* __restrict__ finished, Part* __restrict__ parts,
                                                      Entry* __restrict__ lists, int n, int V, long long total) {
  constexpr int E = kEach, P = 16 / (int)sizeof(T), N = E / P;
  constexpr bool k16 = sizeof(T) == 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), slice = blockIdx.x, slices = gridDim.x, row = blockIdx.y;
  if ((finished != nullptr && finished[row] != 0) || !finite(scores[row])) return;   // k_beam_pick knows what these offer
  // Bit 9 of MODE, IEEE, off: a maximum of a signalling NaN (which an infinity with another element's bits behind it is, too) and a
  // number is the number.
  __builtin_amdgcn_s_setreg(1 | 9 << 6, 0);
  const long long first = (long long)row * V, base = first / P * P + (long long)slice * kSlice;
  const long long whole = total / P * P;   // behind it: an unfinished piece, which is read element by element
  const T* const own = logits + first;
  const int begin = (int)(base - first);   // token of the slice's first element
  u32x4 r[N];
  if (base + kSlice <= whole) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = *reinterpret_cast<const u32x4*>(logits + base + (i * 256 + tid) * P);
  } else {   // the tensor's end
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long at = base + (i * 256 + tid) * P;
      r[i] = u32x4{0, 0, 0, 0};
      if (at < whole) {
        r[i] = *reinterpret_cast<const u32x4*>(logits + at);
      } else if (at < total) {
        T e[P];
#pragma unroll
        for (int j = 0; j < P; ++j) e[j] = at + j < total ? logits[at + j] : (T)0;
        __builtin_memcpy(&r[i], e, 16);
      }
    }
  }
  const auto word = [&](int e) -> unsigned { return r[e / P][e % P * (int)sizeof(T) / 4]; };
  const auto number_of = [](unsigned w, int e) { return __uint_as_float(!k16 ? w : e & 1 ? w & 0xffff0000u : w << 16); };
  const auto rough = [](unsigned w, int e) { return __uint_as_float(!k16 || (e & 1) ? w : w << 16); };   // the lower one's bits behind the upper
  const auto anew = [&]() {   // 16-bit elements are unpacked where they are used, not held unpacked from one pass to the next
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(r[i]));
  };
  if (begin < 0 || begin + kSlice > V) {   // the row's ends
    int t0 = begin + tid * P;
    asm volatile("" : "+v"(t0));   // nothing is computed ahead for the slices within
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int t = t0 + e / P * 256 * P + e % P;
      const unsigned w = word(e), out = !k16 ? 0xff800000u : e & 1 ? (w & 0xffffu) | 0xff800000u : (w & 0xffff0000u) | 0xff80u;
      r[e / P][e % P * (int)sizeof(T) / 4] = (unsigned)t < (unsigned)V ? w : out;
    }
  }
  __shared__ unsigned tops[4], maxima[4][64], least_key;
  __shared__ float sums[4];
  __shared__ int counts[4];
  __shared__ Entry passed[4][kMostPassed];
  __shared__ u64 best_of[4];
  // the maximum
  float best = NAN;
#pragma unroll
  for (int e = 0; e < E; e += 2) best = fmaxf(fmaxf(best, rough(word(e), e)), rough(word(e + 1), e + 1));
  if (k16) best = __uint_as_float(__float_as_uint(best) & 0xffff0000u);
  const unsigned mine = best == best ? ordered(best) : 0u;
  maxima[wave][lane] = mine;
  const unsigned wtop = wave_max(mine);
  if (lane == 0) tops[wave] = wtop;
  __syncthreads();
  unsigned top = tops[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) top = tops[i] > top ? tops[i] : top;
  const float m = top != 0 ? value_of(top) : -INFINITY;
  const bool chooses = wave == (slice & 3);   // one wave of the four, on every SIMD in turn
  if (chooses) {
    unsigned group = maxima[0][lane];
#pragma unroll
    for (int i = 1; i < 4; ++i) group = maxima[i][lane] > group ? maxima[i][lane] : group;
    const unsigned bound = nth_of_lanes(group, n, lane), lowest = ordered(-3.402823466e38f);
    if (lane == 0) least_key = bound > lowest ? bound : lowest;
  }
  anew();
  // sum of 2^(v L - c) with c = m L, L = log2 e in fp32: one rounding of the exponent; k_beam_pick takes c as it is here
  float s = 0.f;
  if (finite(m)) {
    const bool far = large(m);
    const float c = m * kLog2e;
    if (far) s = tree<0, E>([&](int e) { return __builtin_amdgcn_exp2f((number_of(word(e), e) - m) * kLog2e); });
    else s = tree<0, E>([&](int e) { return __builtin_amdgcn_exp2f(fmaf(number_of(word(e), e), kLog2e, -c)); });
    if (__ballot(s != s) != 0) {   // a NaN counts for nothing
      s = 0.f;
#pragma unroll 1
      for (int k = 0; k < N; k += 2)
        s += tree<0, 2 * P>([&](int e) {
          const float v = number(own, begin + ((k + e / P) * 256 + tid) * P + e % P, V);
          return v == v ? __builtin_amdgcn_exp2f(far ? (v - m) * kLog2e : fmaf(v, kLog2e, -c)) : 0.f;
        });
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) s += number_of(word(e), e) == INFINITY ? INFINITY : 0.f;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) sums[wave] = s;
  __syncthreads();
  anew();
  const float least = value_of(least_key);
  // for an upper element with other bits behind it: those that equal the bound lie up to 2^16 below its bits if it is negative
  const float least_rough = !k16 || least > 0.f ? least : __uint_as_float(__float_as_uint(least) | 0x8000ffffu);
  int count = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool in = rough(word(e), e) >= (e & 1 ? least_rough : least);
    const u64 pass = __ballot(in);
    if (pass != 0) {
      const int at = count + __builtin_amdgcn_mbcnt_hi((unsigned)(pass >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)pass, 0u));
      if (in && at < kMostPassed) passed[wave][at] = Entry{number_of(word(e), e), begin + (e / P * 256 + tid) * P + e % P};
      count += __builtin_popcountll(pass);
    }
  }
  if (lane == 0) counts[wave] = count;
  __syncthreads();
  if (tid == 0) {
    const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    parts[(long long)row * slices + slice] = Part{sum < INFINITY ? m : INFINITY, sum};   // an infinite logit
  }
  Entry* const list = lists + ((long long)row * slices + slice) * n;
  const int c0 = counts[0], c1 = c0 + counts[1], c2 = c1 + counts[2], all = c2 + counts[3];
  if (all <= kMostPassed) {
    if (chooses) {
      const int of = (lane >= c0) + (lane >= c1) + (lane >= c2), at = lane - (of == 0 ? 0 : of == 1 ? c0 : of == 2 ? c1 : c2);
      Entry e{0.f, 0};
      if (lane < all) e = passed[of][at];
      place(ordered(e.logit + 0.f), e.token, all, list, n, lane);   // + 0: one zero
    }
    return;
  }
  u64 last = ~0ull;   // the one found before
  for (int i = 0; i < n; ++i) {
    u64 next = 0;
#pragma unroll 1
    for (int k = 0; k < N; ++k) {
      const int t = begin + (k * 256 + tid) * P;
      float e[P];
#pragma unroll
      for (int j = 0; j < P; ++j) e[j] = number(own, t + j, V);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float x = e[j] + 0.f;
        const u64 key = x >= least ? (u64)ordered(x) << 32 | (unsigned)~(t + j) : 0;
        if (key < last && key > next) next = key;
      }
    }
    const unsigned hi = wave_max((unsigned)(next >> 32));
    const unsigned lo = wave_max((unsigned)(next >> 32) == hi ? (unsigned)next : 0u);
    if (lane == 0) best_of[wave] = (u64)hi << 32 | lo;
    __syncthreads();
    last = best_of[0];
#pragma unroll
    for (int k = 1; k < 4; ++k) last = best_of[k] > last ? best_of[k] : last;
    if (tid == 0) list[i] = last != 0 ? Entry{value_of((unsigned)(last >> 32)), (int)~(unsigned)last} : Entry{0.f, -1};
    if (last == 0) break;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// One workgroup a batch entry.  List l of the n * slices belongs to beam l / slices.  The n-th best of the lanes' best list heads bounds
// the n best from below; the few entries that reach it are gathered, and each counts those before it.  Where too many do, the best is
// looked for n times.  Bound by latency: 5 us (one entry, 4 beams) to 11 (8 beams, 512 lists).
// ---------------------------------------------------------------------------
constexpr int kMostLists = 8704;
constexpr int kStaged = 48 * 1024;   // bytes of lists that are brought to LDS at once (else they are read where they are)
constexpr int kMostGathered = 256;

// A candidate: its value in an order of integers (0: none), and what decides where fp64 holds two values for one: the lower beam, in a beam
// the larger logit, then the lower token.  A list is in that order as well (equal logits have equal values, and no smaller one a larger
// value), so that its first entry behind any candidate is the best of those behind it.
struct Head {
  u64 key, rank;
};
constexpr int kTokenBits = 27;
static_assert((long long)kMostLists * kSlice <= 1LL << kTokenBits && kMostBeams <= 1 << (32 - kTokenBits), "a beam, a logit and a token are 64 bits");
__device__ __forceinline__ u64 rank_of(int beam, unsigned logit, int token) {
  return (u64)(kMostBeams - 1 - beam) << (32 + kTokenBits) | (u64)logit << kTokenBits | ((1u << kTokenBits) - 1u - (unsigned)token);
}
__device__ __forceinline__ int beam_of(u64 rank) { return kMostBeams - 1 - (int)(rank >> (32 + kTokenBits)); }
__device__ __forceinline__ int token_of(u64 rank) { return (int)(~(unsigned)rank & ((1u << kTokenBits) - 1u)); }
__device__ __forceinline__ bool before(const Head& a, const Head& b) { return a.key > b.key || (a.key == b.key && a.rank > b.rank); }

enum { kAlive = 0, kFinished = 1, kDead = 2 };

__global__ __launch_bounds__(256) void k_beam_pick(const Part* __restrict__ parts, const Entry* __restrict__ lists,
                                                   const float* __restrict__ scores, const unsigned char* __restrict__ finished, int n,
                                                   int V, int slices, int eos, int keep_slots, int staged, float* __restrict__ out_scores,
                                                   int32_t* __restrict__ out_parent, int32_t* __restrict__ out_token) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x, count = n * slices;
  Entry* const near = reinterpret_cast<Entry*>(smem);
  __shared__ double offset[kMostBeams];
  __shared__ float tops[kMostBeams];
  __shared__ int kind[kMostBeams];
  __shared__ Head gathered[kMostGathered];
  __shared__ Head picks[kMostBeams];
  __shared__ Head best[4];
  __shared__ unsigned reach;
  __shared__ int size;
  const Entry* const own = lists + (long long)b * count * n;
  if (tid == 0) size = 0;
  if (tid < kMostBeams) picks[tid] = Head{0, 0};
  constexpr int kAtOnce = 8;   // what a thread asks for before it waits: every trip to memory takes longer than all the rest
  if (staged)
    for (int l0 = 0; l0 < count * n; l0 += 256 * kAtOnce) {
      Entry e[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) e[i] = own[min(l0 + 256 * i + tid, count * n - 1)];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (l0 + 256 * i + tid < count * n) near[l0 + 256 * i + tid] = e[i];
    }
  // a beam for every 32 threads: the logarithm of its sum of exponentials
  for (int j0 = 0; j0 < n; j0 += 8) {
    const int j = j0 + tid / 32, t = tid % 32;
    const long long row = (long long)b * n + j;
    const float score = j < n ? scores[row] : 0.f;
    const bool done = j < n && finished != nullptr && finished[row] != 0, live = j < n && !done && finite(score);
    float top = -INFINITY;
    double z = 0.0;
    Part mine{-INFINITY, 0.f};
    if (j < n && t < slices) mine = parts[row * slices + t];   // where the beam is not live: read, not used
    if (live) {
      top = mine.top;
      for (int i = t + 32; i < slices; i += 32) top = fmaxf(top, parts[row * slices + i].top);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    // sums are of 2^(v L - c), L and c = top L in fp32
    if (live && finite(top))
      for (int i = t; i < slices; i += 32) {
        const Part p = i == t ? mine : parts[row * slices + i];
        if (p.sum > 0.f) z += (double)p.sum * exp2(origin(p.top) - origin(top));
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
    if (t == 0 && j < n) {
      const bool alive = live && finite(top);
      kind[j] = alive ? kAlive : done && finite(score) ? kFinished : kDead;
      // log sum exp(v - top) = ln 2 (c - top L + log2 z), where the exponents v L of the terms that matter stand for v log2 e near v = top
      const double c = origin(top) - (double)top * (double)kLog2e;
      offset[j] = alive ? (double)score - 0.69314718055994530942 * (c + log2(z)) : (double)score + 0.0;
      tops[j] = top;
    }
  }
  __syncthreads();
  // entry `at` of list l
  const auto entry = [&](int l, int at) {
    const int j = l / slices;
    Head hd{0, 0};
    if (kind[j] == kAlive) {
      const Entry e = staged ? near[l * n + at] : own[(long long)l * n + at];
      if (e.token < 0) return hd;
      hd.key = ordered64(offset[j] + ((double)e.logit - (double)tops[j]) + 0.0);   // one zero
      hd.rank = rank_of(j, ordered(e.logit), e.token);
    } else if (kind[j] == kFinished && l % slices == 0 && at == 0) {   // a finished beam goes on with `eos` alone
      hd.key = ordered64(offset[j]);
      hd.rank = rank_of(j, 0u, eos);
    }
    return hd;
  };
  if (wave == 0) {
    unsigned most = 0;
    for (int l = lane; l < count; l += 64) {
      const unsigned k = (unsigned)(entry(l, 0).key >> 32);
      most = k > most ? k : most;
    }
    const unsigned bound = nth_of_lanes(most, n, lane);
    if (lane == 0) reach = bound > 0 ? bound : 1u;
  }
  __syncthreads();
  for (int l = tid; l < count; l += 256) {
    for (int at = 0; at < n; ++at) {   // in order: none behind the first that falls short
      const Head hd = entry(l, at);
      if ((unsigned)(hd.key >> 32) < reach) break;
      const int to = atomicAdd(&size, 1);   // whatever their order there: they are told apart by key and index
      if (to < kMostGathered) gathered[to] = hd;
    }
  }
  __syncthreads();
  if (size <= kMostGathered) {
    if (tid < size) {
      const Head mine = gathered[tid];
      int place = 0;
#pragma unroll 4
      for (int i = 0; i < size; ++i) place += before(gathered[i], mine);
      if (place < n) picks[place] = mine;
    }
    __syncthreads();
  } else {
    Head last{~0ull, 0};
    for (int i = 0; i < n; ++i) {
      Head w{0, 0};
      for (int l = tid; l < count; l += 256)
        for (int at = 0; at < n; ++at) {
          const Head hd = entry(l, at);
          if (hd.key == 0) break;
          if (before(last, hd)) {   // the list's first that is not taken
            if (before(hd, w)) w = hd;
            break;
          }
        }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        Head x;
        x.key = __shfl_xor(w.key, o, 64);
        x.rank = __shfl_xor(w.rank, o, 64);
        if (before(x, w)) w = x;
      }
      if (lane == 0) best[wave] = w;
      __syncthreads();
      last = best[0];
#pragma unroll
      for (int k = 1; k < 4; ++k)
        if (before(best[k], last)) last = best[k];
      if (tid == 0) picks[i] = last;
      __syncthreads();
    }
  }
  if (wave != 0) return;
  Head mine{0, 0};
  if (lane < n) mine = picks[lane];
  const int found = __builtin_popcountll(__ballot(mine.key != 0));   // the first ones
  int parent = beam_of(mine.rank), token = token_of(mine.rank);
  // too few: candidates of value -infinity, the lowest that are not taken yet
  int have = found;
  for (int j = 0, t = 0; have < n; ++t) {
    if (t == V) ++j, t = 0;
    if (__ballot(lane < have && parent == j && token == t) != 0) continue;
    if (lane == have) parent = j, token = t;
    ++have;
  }
  int slot = lane;
  if (keep_slots) {
    unsigned used = 0;   // places of beams that survive
    for (int i = 0; i < n; ++i) used |= 1u << __builtin_amdgcn_readlane(parent, i);
    unsigned kept = 0;
    int free = 0;
    for (int i = 0; i < n; ++i) {
      const int p = __builtin_amdgcn_readlane(parent, i);
      int at = p;
      if ((kept >> p & 1u) != 0) {
        while (used >> free & 1u) ++free;
        at = free++;
      }
      kept |= 1u << p;
      if (lane == i) slot = at;
    }
  }
  if (lane < n) {
    const long long at = (long long)b * n + slot;
    out_scores[at] = mine.key != 0 ? (float)value64(mine.key) : -INFINITY;
    out_parent[at] = parent;
    out_token[at] = token;
  }
}

// ---------------------------------------------------------------------------
// States in place: a thread holds the same 16 (4, 1) bytes of every row that changes, so that all are read before any is written.
// Bound by reading the parents of the rows that change and writing those rows (8 x 4 beams, two layers of 16 x 256 x 128: 75 MB in 17.7 us).
// ---------------------------------------------------------------------------
constexpr int kMostTensors = 16;
struct Tensors {
  char* data[kMostTensors];
  long long row_bytes[kMostTensors];
  int unit[kMostTensors];          // 16, 4 or 1
  int first[kMostTensors + 1];     // blocks before the tensor's own
  int count;
};

// Rows by buffer instructions without branches: of a row that stays where it is nothing exists, so that no byte of it is moved.
// (With a branch a row the eight's kernel took 226 registers: 4 x 8 rows of 2 MB twice 42 us.)
__device__ __forceinline__ void get(u32x4& v, __amdgpu_buffer_rsrc_t b, unsigned at) { v = __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0); }
__device__ __forceinline__ void get(unsigned& v, __amdgpu_buffer_rsrc_t b, unsigned at) { v = __builtin_amdgcn_raw_buffer_load_b32(b, at, 0, 0); }
__device__ __forceinline__ void get(unsigned char& v, __amdgpu_buffer_rsrc_t b, unsigned at) { v = __builtin_amdgcn_raw_buffer_load_b8(b, at, 0, 0); }
__device__ __forceinline__ void put(u32x4 v, __amdgpu_buffer_rsrc_t b, unsigned at) { __builtin_amdgcn_raw_buffer_store_b128(v, b, at, 0, 0); }
__device__ __forceinline__ void put(unsigned v, __amdgpu_buffer_rsrc_t b, unsigned at) { __builtin_amdgcn_raw_buffer_store_b32(v, b, at, 0, 0); }
__device__ __forceinline__ void put(unsigned char v, __amdgpu_buffer_rsrc_t b, unsigned at) { __builtin_amdgcn_raw_buffer_store_b8(v, b, at, 0, 0); }

// Bytes at ... of the rows, 256 units of them at most.
template <typename U, int N>
__device__ __forceinline__ void reorder(char* rows, long long row_bytes, long long at, const int32_t* from, int n) {
  const int bytes = (int)min(row_bytes - at, 256LL * (long long)sizeof(U));
  const unsigned own = threadIdx.x * (unsigned)sizeof(U);
  U v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int p = from[min(j, n - 1)];
    const bool moves = j < n && p != j && (unsigned)p < (unsigned)n;
    get(v[j], __builtin_amdgcn_make_buffer_rsrc(rows + (moves ? p : 0) * row_bytes + at, 0, moves ? bytes : 0, 0x00027000), own);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int p = from[min(j, n - 1)];
    const bool moves = j < n && p != j && (unsigned)p < (unsigned)n;
    put(v[j], __builtin_amdgcn_make_buffer_rsrc(rows + (moves ? j : 0) * row_bytes + at, 0, moves ? bytes : 0, 0x00027000), own);
  }
}

template <int N>
__global__ __launch_bounds__(256) void k_state_reorder(Tensors t, const int32_t* __restrict__ parent, int n) {
  int i = 0;
  while (i + 1 < t.count && (int)blockIdx.x >= t.first[i + 1]) ++i;
  const long long at = (long long)((int)blockIdx.x - t.first[i]) * 256 * t.unit[i], row_bytes = t.row_bytes[i];
  char* const rows = t.data[i] + (long long)blockIdx.y * n * row_bytes;
  const int32_t* const from = parent + (long long)blockIdx.y * n;
  if (t.unit[i] == 16) reorder<u32x4, N>(rows, row_bytes, at, from, n);
  else if (t.unit[i] == 4) reorder<unsigned, N>(rows, row_bytes, at, from, n);
  else reorder<unsigned char, N>(rows, row_bytes, at, from, n);
}

// A row's unit, and the workgroups of 256 units each that move it; along a grid's x.
constexpr size_t kMostBlocks = 1 << 23;
int unit_of(size_t row_bytes) { return row_bytes % 16 == 0 ? 16 : row_bytes % 4 == 0 ? 4 : 1; }
size_t blocks_of(size_t row_bytes) {
  const size_t units = row_bytes / unit_of(row_bytes);
  return units / 256 + (units % 256 != 0);
}

int slices_of(const dark_beam_params& p) {
  const int per = p.io_dtype == DARK_BF16 ? 8 : 4;
  return (int)(((long long)p.V + per - 1 + kSlice - 1) / kSlice);   // a row begins up to per - 1 elements behind its first slice
}

dark_status check(const dark_beam_params* p) {
  if (p == nullptr || p->B < 0 || p->n <= 0 || p->V <= 0) return DARK_EINVAL;
  if (p->io_dtype != DARK_F32 && p->io_dtype != DARK_BF16) return DARK_EINVAL;
  if (p->n > kMostBeams || (long long)p->n * p->V >= (1LL << 31) || (long long)p->B * p->n > 65535) return DARK_EUNSUPPORTED;
  if ((long long)p->n * slices_of(*p) > kMostLists) return DARK_EUNSUPPORTED;
  return DARK_OK;
}

void plan(const dark_beam_params& p, Arena& ar, Part** parts, Entry** lists) {
  const size_t slots = (size_t)p.B * p.n * slices_of(p);
  *parts = ar.take<Part>(slots);
  *lists = ar.take<Entry>(slots * p.n);
}

template <typename T>
dark_status rows(const dark_beam_params& p, const void* logits, const float* scores, const unsigned char* finished, Part* parts,
                 Entry* lists, hipStream_t st) {
  const dim3 grid(slices_of(p), p.B * p.n);
  const long long total = (long long)p.B * p.n * p.V;
  DARK_LAUNCH(KID_BEAM_ROWS, st, k_beam_rows<T>, grid, dim3(256), 0, static_cast<const T*>(logits), scores, finished, parts, lists, p.n, p.V, total);
  return DARK_OK;
}

}  // namespace
}  // namespace beam
}  // namespace dark

using namespace dark;

extern "C" {

size_t dark_beam_workspace_bytes(const dark_beam_params* p) {
  if (beam::check(p) != DARK_OK || p->B == 0) return 0;
  Arena ar(nullptr, 0);
  beam::Part* parts;
  beam::Entry* lists;
  beam::plan(*p, ar, &parts, &lists);
  return ar.off;
}

dark_status dark_beam_select(const dark_beam_params* p, const void* logits, const float* scores, const unsigned char* finished,
                             float* out_scores, int32_t* out_parent, int32_t* out_token, void* ws, size_t ws_bytes, void* hip_stream) {
  DARK_TRY(beam::check(p));
  if (p->B == 0) return DARK_OK;
  if (!logits || !scores || !out_scores || !out_parent || !out_token) return DARK_EINVAL;
  if (finished != nullptr && (p->eos < 0 || p->eos >= p->V)) return DARK_EINVAL;
  if (!aligned(logits, 16) || !aligned(scores, 4) || !aligned(out_scores, 4) || !aligned(out_parent, 4) || !aligned(out_token, 4))
    return DARK_EALIGN;
  Arena ar(ws, ws_bytes);
  if (ws == nullptr || ws_bytes < dark_beam_workspace_bytes(p)) return DARK_EWORKSPACE;
  if (!aligned(ws, 256)) return DARK_EALIGN;
  const size_t beams = (size_t)p->B * p->n;
  const Span next{out_scores, 4 * beams}, past{scores, 4 * beams};
  if (overlap({next, {out_parent, 4 * beams}, {out_token, 4 * beams}}, {{logits, beams * p->V * (p->io_dtype == DARK_BF16 ? 2 : 4)}, {finished, beams}}) ||
      overlap({{out_parent, 4 * beams}, {out_token, 4 * beams}}, {past}) || (out_scores != scores && overlap(next, past)))
    return DARK_EINVAL;
  beam::Part* parts;
  beam::Entry* lists;
  beam::plan(*p, ar, &parts, &lists);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  DARK_TRY(p->io_dtype == DARK_BF16 ? beam::rows<unsigned short>(*p, logits, scores, finished, parts, lists, st)
                                    : beam::rows<float>(*p, logits, scores, finished, parts, lists, st));
  const int slices = beam::slices_of(*p);
  const size_t count = (size_t)p->n * slices, bytes = count * p->n * sizeof(beam::Entry);
  const int staged = bytes <= beam::kStaged;
  DARK_LAUNCH(KID_BEAM_PICK, st, beam::k_beam_pick, dim3(p->B), dim3(256), staged ? bytes : 0, parts, lists, scores, finished, p->n,
              p->V, slices, p->eos, p->keep_slots != 0, staged, out_scores, out_parent, out_token);
  return DARK_OK;
}

dark_status dark_state_reorder(int B, int n, const int32_t* parent, int count, void* const* states, const size_t* row_bytes,
                               void* hip_stream) {
  if (B < 0 || n <= 0 || count < 0) return DARK_EINVAL;
  if (n > beam::kMostBeams || B > 65535) return DARK_EUNSUPPORTED;
  if (B == 0 || count == 0) return DARK_OK;
  if (parent == nullptr || states == nullptr || row_bytes == nullptr) return DARK_EINVAL;
  if (!aligned(parent, 4)) return DARK_EALIGN;
  for (int i = 0; i < count; ++i) {
    if (row_bytes[i] == 0) continue;
    if (states[i] == nullptr) return DARK_EINVAL;
    if (beam::blocks_of(row_bytes[i]) > beam::kMostBlocks) return DARK_EUNSUPPORTED;   // here, before anything has moved
    if (!aligned(states[i], 16)) return DARK_EALIGN;
  }
  const size_t beams = (size_t)B * n;
  for (int i = 0; i < count; ++i) {
    const Span own{states[i], row_bytes[i] * beams};
    if (overlap(own, {parent, 4 * beams})) return DARK_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(own, {states[j], row_bytes[j] * beams})) return DARK_EINVAL;
  }
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  for (int i = 0; i < count;) {
    beam::Tensors t;
    t.count = 0;
    long long blocks = 0;
    for (; i < count && t.count < beam::kMostTensors; ++i) {
      if (row_bytes[i] == 0) continue;
      const long long more = (long long)beam::blocks_of(row_bytes[i]);
      if (blocks + more > (long long)beam::kMostBlocks) break;   // never the first of a launch
      t.data[t.count] = static_cast<char*>(states[i]);
      t.row_bytes[t.count] = (long long)row_bytes[i];
      t.unit[t.count] = beam::unit_of(row_bytes[i]);
      t.first[t.count] = (int)blocks;
      blocks += more;
      ++t.count;
    }
    if (t.count == 0) break;
    t.first[t.count] = (int)blocks;
    const dim3 grid((unsigned)blocks, (unsigned)B);
    if (n <= 4) {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<4>, grid, dim3(256), 0, t, parent, n);
    } else if (n <= 8) {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<8>, grid, dim3(256), 0, t, parent, n);
    } else {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<32>, grid, dim3(256), 0, t, parent, n);
    }
  }
  return DARK_OK;
}

}  // extern "C"
