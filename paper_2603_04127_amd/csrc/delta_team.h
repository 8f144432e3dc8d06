// The gated delta rule's scans with a wave for each row tile of 16 columns of the state (see delta_scan.h for one wave that does all).
//
// A wave by itself takes several cycles for an instruction, whatever it is, where the chunks' states hang on each other; what a SIMD does in that
// time grows with its waves, and a CU with its SIMDs.  So the 16 columns' work is dealt to a team, four waves for bf16's chunks of 64 rows and two for
// fp32's of 32: each has one of the chunk's row tiles and a part of the state's rows.  What a wave has as sums and all need as an operand goes
// through LDS: the state's planes, R, and U, with a barrier behind each.  bf16 rows that fill the tiles are brought by two waves and loads that end in
// LDS (DIRECT), a part between two barriers: a whole chunk's at once, six instructions each, kept their wave from the first barrier for a third of the
// chunk.  All others go through the registers of eight waves (of four, with as long between the same barriers: 5 to 13 % more; four where fp32 rows of
// 128 leave no registers for eight).
// One wave and a team, DIRECT: prompt of 16 x 777 x 128 44 -> 26 us, prefill of 64 x 8192 x 128 425 -> 364, 16 x 2048 of 128 and 256 columns 103 -> 64, training of
// 24 x 4096 x 64 forward 145 -> 92, backward 169 -> 102 (two waves a team, with all loads at once: no faster than one).  Through registers: heads of 100 and 128 for
// that prompt 46 -> 39, 8 heads of 1000 x 96 and 80 backward 63 -> 41; fp32, 8 heads of 1000 x 64 64 -> 54, backward 69 -> 55.
// What is not DIRECT adds up in the same order here and there, so that a sequence's results do not depend on how many others there are.
#pragma once

#include "delta_scan.h"

namespace dark {
namespace delta {

// Half of an operand: what a tile's four values of a lane are in it.
template <int N>
struct Half {
  u32x2 p[N];
};
template <int N>
__device__ static inline Half<N> split_half(f32x4 a) {
  const Planes<N> f = split<N>(a, a);
  Half<N> h;
#pragma unroll
  for (int p = 0; p < N; ++p) h.p[p] = u32x2{f.p[p][0], f.p[p][1]};
  return h;
}

// Operands in LDS for two chunks, or, of those that go straight there, for one what is needed late in a chunk: P forward, Q and T backward.
template <typename T_, int D1, int TEAMS, int NP, bool REV, bool DIRECT>
struct TeamChunks {
  typedef T_ T;
  static constexpr int C = Kind<T>::kChunk, NI = Kind<T>::kIn, NB = blocks_of(C), VC = 16 * TEAMS, KS = D1 / 32;
  static constexpr bool kDirect = DIRECT;
  static constexpr int kTeam = C / 16, kOwn = D1 / 16 / kTeam;   // waves of a team, tiles of the state of each
  static constexpr int kLoaders = kDirect ? 2 : NI == 3 && D1 > 64 ? 4 : 8, kThreads = 64 * (kTeam * TEAMS + kLoaders), NTH = 64 * kLoaders;
  typedef Mat<C, D1, NI> MK;
  typedef Mat<C, VC, NI> MV;
  static constexpr int kQ = NP > 0 ? MK::kAll : 0, kV = MV::kAll, kW = kScanVecs * C * 4, kT = 3 * NB * 1024, kP = NP * NB * 1024;
  static constexpr int qs = kDirect && REV ? 1 : 2, ts = kDirect && REV ? 1 : 2, ps = kDirect && !REV ? 1 : 2;   // buffers
  static constexpr int k = 0, q = 2 * MK::kAll, v = q + qs * kQ, w = v + 2 * kV, t = w + 2 * kW, p = t + ts * kT, x = p + ps * kP;
  // exchange, of a team: the state's planes, in their place later U's (those of the update, and those of P U or of dO); R's
  static constexpr int NS = C / 32, kRows = 3 * 1024 * NS, kMore = REV ? kRows : NP * 1024 * NS;
  static constexpr int kFirst = KS * 3 * 1024, kLast = kRows + kMore, x2 = kFirst > kLast ? kFirst : kLast, kX = x2 + kRows;
  static constexpr int all = x + TEAMS * kX;
  static_assert(all <= 160 * 1024, "fits the LDS");
};

// Four loads of 1 KB that end in LDS one behind the other, at `off[i]` behind `base` in memory.  The instruction's own offset counts in memory and in
// LDS, so the second to fourth need neither their own m0 nor their own address: two instructions a KB instead of six.  `off[i]` is less by i KB.
// (See dma16_to_lds for the wait states.)
__device__ static inline void dma64_to_lds(const void* base, const unsigned (&off)[4], int to) {
  const unsigned dst = __builtin_amdgcn_readfirstlane((unsigned)to);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)base), hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)base >> 32));
  asm volatile(
      "s_mov_b32 m0, %5\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %4 offset:0x400\n\t"
      "global_load_lds_dwordx4 %2, %4 offset:0x800\n\tglobal_load_lds_dwordx4 %3, %4 offset:0xc00" ::"v"(off[0]),
      "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"((unsigned long long)hi << 32 | lo), "s"(dst)
      : "memory", "m0");
}
// C rows of a tile whose rows they fill.  A wave's lanes write where they lie, so that a lane asks for the 16 bytes that the swizzle puts
// there.  Rows behind the last are copies of it (their weights are 0: k_delta_prep).
template <int C, int D>
struct Tile {
  typedef Mat<C, D, 1> M;
  static constexpr int kLanes = M::RB / 16, kRows = 64 / kLanes, kLoads = C / kRows;   // lanes a row, rows a load, loads
  static constexpr bool kFour = kLoads % 4 == 0;
  static_assert(4 * kRows % 16 == 0, "the swizzle repeats every 16 rows");
  unsigned off[4];
  __device__ Tile(const Rows& x, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * kRows + lane / kLanes;
      off[i] = (unsigned)row * x.row + (unsigned)(((lane % kLanes) ^ swz<M::RB>(row & 15)) << 4) - 1024u * i;   // a row is kLanes * 16 bytes or more
    }
  }
  __device__ void load(int tile, const Rows& x, int r0, int nr, int lane) const {
    const char* const first = x.head + (long long)r0 * x.row;
    if (kFour && nr == C) {
#pragma unroll
      for (int i = 0; i < kLoads; i += 4) dma64_to_lds(first + (long long)(i * kRows) * x.row, off, tile + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = i * kRows + lane / kLanes;
        dma16_to_lds(first, (unsigned)min(row, nr - 1) * x.row + (unsigned)(((lane % kLanes) ^ swz<M::RB>(row & 15)) << 4), reinterpret_cast<void*>((uintptr_t)(tile + i * 1024)));
      }
    }
  }
};
// KB as they are.
template <int KB>
__device__ static inline void copy_to_lds(int tile, const void* from, int lane) {
  const unsigned own = (unsigned)lane * 16u, off[4] = {own, own, own, own};
#pragma unroll
  for (int i = 0; i < KB; ++i) {
    if (i % 4 == 0 && i + 4 <= KB) dma64_to_lds(static_cast<const char*>(from) + i * 1024, off, tile + i * 1024);
    else if (i >= KB / 4 * 4) dma16_to_lds(static_cast<const char*>(from) + i * 1024, own, reinterpret_cast<void*>((uintptr_t)(tile + i * 1024)));
  }
}

// The loading waves.  A chunk's barriers stand behind the state's planes, R, U, and the last reads.  A single buffer's operands are there before the
// second (T backward) or the third (P, Q), the next chunk's before the last.
template <typename L, int D1, int NP, bool REV>
__device__ static inline void load_keys(const Args& A, int bh, int n, int lane) {
  constexpr int C = L::C, N = L::MK::kAll / 1024;
  const Rows xk = rows_at<unsigned short>(A.K, A, bh, A.dk, n, 0, A.dk), xq = rows_at<unsigned short>(A.Q, A, bh, A.dk, n, 0, A.dk);
  const Tile<C, D1> tile(xk, lane);   // K's rows and Q's lie alike
  const int chunks = (n + C - 1) / C;
  const auto keys = [&](int i) {
    const int r0 = (REV ? chunks - 1 - i : i) * C;
    tile.load(L::k + (i & 1) * L::MK::kAll, xk, r0, min(C, n - r0), lane);
  };
  const auto queries = [&](int i) {
    const int r0 = (REV ? chunks - 1 - i : i) * C;
    tile.load(L::q + (REV ? 0 : i & 1) * L::kQ, xq, r0, min(C, n - r0), lane);
  };
  keys(0);
  if (NP > 0 && !REV) queries(0);
  wait_vmcnt0();
  lds_barrier();
  for (int i = 0; i < chunks; ++i) {
    const bool more = i + 1 < chunks;
    if (REV) queries(i);
    else if (more) keys(i + 1);
    lds_barrier();
    if (more) {
      if (REV) keys(i + 1);
      else if (NP > 0) queries(i + 1);
    }
    lds_barrier();
    if (REV) {
      if (more) wait_loads<N>();
      else wait_vmcnt0();
    }
    lds_barrier();
    wait_vmcnt0();
    lds_barrier();
  }
}
template <typename L, int D1, int NP, bool REV>
__device__ static inline void load_rest(const Args& A, int bh, const Rows& xv, int n, int lane) {
  constexpr int C = L::C, NB = L::NB;
  const Tile<C, L::VC> tile(xv, lane);
  const int chunks = (n + C - 1) / C;
  const auto chunk = [&](int i) { return REV ? chunks - 1 - i : i; };
  const auto triangle = [&](int i) { copy_to_lds<3 * NB>(L::t + (REV ? 0 : i & 1) * L::kT, (REV ? A.trit : A.tri) + chunk_at(A, bh, chunk(i)) * (3 * NB * 64), lane); };
  const auto weights = [&](int i) { copy_to_lds<NP * NB>(L::p + (REV ? i & 1 : 0) * L::kP, A.pri + chunk_at(A, bh, chunk(i)) * (NP * NB * 64), lane); };
  const auto values = [&](int i) {
    const int r0 = chunk(i) * C;
    copy_to_lds<L::kW / 1024>(L::w + (i & 1) * L::kW, A.vec + chunk_at(A, bh, chunk(i)) * (kVecs * C), lane);
    tile.load(L::v + (i & 1) * L::kV, xv, r0, min(C, n - r0), lane);
  };
  constexpr int kNext = (L::kW + L::kV + (REV ? L::kP : L::kT)) / 1024;
  values(0);
  if (REV) weights(0);
  else triangle(0);
  wait_vmcnt0();
  lds_barrier();
  for (int i = 0; i < chunks; ++i) {
    const bool more = i + 1 < chunks;
    if (REV) triangle(i);
    else if (NP > 0) weights(i);
    lds_barrier();
    if (more) {
      values(i + 1);
      if (REV) weights(i + 1);
      else triangle(i + 1);
    }
    if (REV) {
      if (more) wait_loads<kNext>();
      else wait_vmcnt0();
    }
    lds_barrier();
    if (!REV) {
      if (more) wait_loads<kNext>();
      else wait_vmcnt0();
    }
    lds_barrier();
    wait_vmcnt0();
    lds_barrier();
  }
}

// Through registers: between the first barrier and the second the next chunk's operands go to LDS, and those of the chunk behind it are asked for.
template <typename L, int D1, int NP, bool VEC, bool REV>
__device__ static inline void load_through(const Args& A, int bh, const Rows& xv, int n, int tid) {
  typedef typename L::T T;
  constexpr int C = L::C, NB = L::NB, NTH = L::NTH;
  const Rows xk = rows_at<T>(A.K, A, bh, A.dk, n, 0, A.dk), xq = rows_at<T>(A.Q, A, bh, A.dk, n, 0, A.dk);
  const u32x4* const tri = REV ? A.trit : A.tri;
  const int chunks = (n + C - 1) / C;
  Load<T, C, D1, NTH, VEC> lk, lq;
  Load<T, C, L::VC, NTH, VEC> lv;
  LoadTri<NB, 3, NTH> lt;
  LoadTri<NB, (NP > 0 ? NP : 1), NTH> lp;
  f32x4 lw = zero4();
  const auto chunk = [&](int i) { return REV ? chunks - 1 - i : i; };
  const auto rows = [&](auto& l, const Rows& x, int i) __attribute__((always_inline)) { l.load(x, chunk(i) * C, min(C, n - chunk(i) * C), tid); };
  const auto keys = [&](int i) __attribute__((always_inline)) { rows(lk, xk, i); };
  const auto queries = [&](int i) __attribute__((always_inline)) { if (NP > 0) rows(lq, xq, i); };
  const auto values = [&](int i) __attribute__((always_inline)) {
    rows(lv, xv, i);
    if (tid < C) lw = reinterpret_cast<const f32x4*>(A.vec + chunk_at(A, bh, chunk(i)) * (kVecs * C))[tid];
  };
  const auto triangles = [&](int i) __attribute__((always_inline)) {
    lt.load(tri + chunk_at(A, bh, chunk(i)) * (3 * NB * 64), tid);
    if (NP > 0) lp.load(A.pri + chunk_at(A, bh, chunk(i)) * (NP * NB * 64), tid);
  };
  const auto put_keys = [&](int buf) __attribute__((always_inline)) { lk.template store<typename L::MK>(L::k + buf * L::MK::kAll, tid); };
  const auto put_queries = [&](int buf) __attribute__((always_inline)) { if (NP > 0) lq.template store<typename L::MK>(L::q + buf * L::kQ, tid); };
  const auto put_values = [&](int buf) __attribute__((always_inline)) {
    lv.template store<typename L::MV>(L::v + buf * L::kV, tid);
    if (tid < C) lds_put(L::w + buf * L::kW + 16 * tid, lw);
  };
  const auto put_triangles = [&](int buf) __attribute__((always_inline)) {
    lt.store(L::t + buf * L::kT, tid);
    if (NP > 0) lp.store(L::p + buf * L::kP, tid);
  };
  keys(0);
  queries(0);
  values(0);
  triangles(0);
  put_keys(0);
  put_queries(0);
  put_values(0);
  put_triangles(0);
  if (chunks > 1) {
    keys(1);
    queries(1);
    values(1);
    triangles(1);
  }
  lds_barrier();
  for (int i = 0; i < chunks; ++i) {
    const bool next = i + 1 < chunks, more = i + 2 < chunks;
    const int buf = (i + 1) & 1;
    lds_barrier();
    if (next) {
      put_keys(buf);
      put_queries(buf);
      put_values(buf);
      put_triangles(buf);
    }
    if (more) {
      keys(i + 2);
      queries(i + 2);
      values(i + 2);
      triangles(i + 2);
    }
    lds_barrier();
    lds_barrier();
    lds_barrier();
  }
}
template <typename L, int D1, int NP, bool VEC, bool REV>
__device__ static inline void load_team(const Args& A, int bh, const void* values, int col0, int n, int tid) {
  const Rows xv = rows_at<typename L::T>(values, A, bh, A.dv, n, col0, min(A.dv - col0, L::VC));
  if constexpr (L::kDirect) {
    if (tid < 64) load_keys<L, D1, NP, REV>(A, bh, n, tid);
    else load_rest<L, D1, NP, REV>(A, bh, xv, n, tid - 64);
  } else {
    load_through<L, D1, NP, VEC, REV>(A, bh, xv, n, tid);
  }
}

// A lane's bases: those of row tile h, and of the wave's part of the state's rows.
template <typename L, bool REV>
struct TeamBases {
  static constexpr int RB = L::MK::RB, RV = L::MV::RB;
  int rows, query, cols, query_cols, value, vec, row, tri, weights, planes, own, half;
  __device__ TeamBases(Lane l, int lane, int team, int h) {
    rows = L::MK::row_base(l) + h * 16 * RB;
    cols = L::MK::col_base(l) ^ (h * L::kOwn << 5);
    query = rows + L::q;
    query_cols = cols + L::q;
    value = (L::MV::col_base(l) ^ (team << 5)) + h * 16 * RV + L::v;
    vec = 16 * l.g + L::w + 64 * h;
    row = 4 * l.i + L::w + 64 * h;
    // of two steps a lower triangle's row tile has block (h, 0), and (h, 1) behind it; of an upper one (h, 1), and (h, 0) before it
    const int first = L::NS == 1 ? h : REV ? (h < 2 ? 2 * h + 1 : h + 2) : h < 2 ? h : 2 * h - 2;
    tri = 16 * lane + L::t + 1024 * first;
    weights = 16 * lane + L::p + 1024 * first;
    planes = 16 * lane + L::x + team * L::kX;
    own = planes + (L::kOwn > 1 ? h * (L::kOwn / 2) * 3 * 1024 : (h >> 1) * 3 * 1024 + 8 * (h & 1));
    half = planes + 8 * (h & 1);
#pragma unroll
    for (int* p : {&rows, &query, &cols, &query_cols, &value, &vec, &row, &tri, &weights, &planes, &own, &half}) asm("" : "+v"(*p));
  }
};

template <int N>
__device__ static inline void put_half(int at, const Half<N>& f) {
#pragma unroll
  for (int p = 0; p < N; ++p) lds_put(at + 1024 * p, f.p[p]);
}
template <int N>
__device__ static inline Planes<N> get_planes(int at) {
  Planes<N> f;
#pragma unroll
  for (int p = 0; p < N; ++p) f.p[p] = lds_get<u32x4>(at + 1024 * p);
  return f;
}
template <int NB, int M>
__device__ static inline Planes<M> get_block(int at) {
  Planes<M> t;
#pragma unroll
  for (int i = 0; i < M; ++i) t.p[i] = lds_get<u32x4>(at + i * NB * 1024);
  return t;
}
// The four values of a tile's column.
template <typename M, int N>
__device__ static inline f32x4 column(int at) {
  f32x4 x;
#pragma unroll
  for (int p = N - 1; p >= 0; --p) {
    const u32x2 v = lds_get_tr16(at + p * M::kBytes);
    const f32x4 y = {__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
    if (p == N - 1) x = y;
    else x += y;
  }
  return x;
}
// A tile's column to scratch.
__device__ static inline void put_tile(f32x4 v, Buffer b, int row, int stride, int c0, Lane l) {
  const unsigned at = (unsigned)((row + 4 * l.g) * stride + c0 + l.i) * 4u;
#pragma unroll
  for (int j = 0; j < 4; ++j) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[j]), b, at, (unsigned)(j * stride) * 4u, 0);
}
// x + sum_s a_s b_s: one chain (two, and their sum behind them, take longer: instructions count, not what a product waits for).  One step's products behind
// the other's (STEP), or, with one plane on a side, the smallest terms of all first: all operands are there before the first product, one wait.
template <bool STEP, int MA, int MB, int S, int NA, int NB>
__device__ static inline f32x4 mma_steps(const Planes<NA> (&a)[S], const Planes<NB> (&b)[S], f32x4 x) {
  if constexpr (!STEP && (MA == 1 || MB == 1)) {
#pragma unroll
    for (int i = (MA > MB ? MA : MB) - 1; i >= 0; --i)
#pragma unroll
      for (int s = 0; s < S; ++s) x = mma1(a[s].p[MA > 1 ? i : 0], b[s].p[MB > 1 ? i : 0], x);
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s) x = mma_of<MA, MB>(a[s], b[s], x);
  }
  return x;
}
// x + t b for a triangle's block, the smallest terms first, or (STEP) in the order of mma_step (TRANS: b t).
template <bool STEP, bool TRANS, int M, int N>
__device__ static inline f32x4 mma_block(const Planes<M>& t, const Planes<N>& b, f32x4 x) {
  constexpr int W = M > N ? M : N;
  if constexpr (!STEP) return TRANS ? mma(b, t, x) : mma(t, b, x);
#pragma unroll
  for (int i = M - 1; i >= 0; --i)
#pragma unroll
    for (int j = W - 1 - i; j >= 0; --j)
      if (j < N) x = TRANS ? mma1(b.p[j], t.p[i], x) : mma1(t.p[i], b.p[j], x);
  return x;
}
// The computing waves: f(chunk, the buffer of its operands, a constant) for every chunk.
template <bool REV, typename F>
__device__ static inline void each_chunk_of_team(int chunks, const F& f) {
  lds_barrier();
  for (int i = 0; i < chunks;) {
    f(REV ? chunks - 1 - i : i, std::integral_constant<int, 0>());
    if (++i == chunks) break;
    f(REV ? chunks - 1 - i : i, std::integral_constant<int, 1>());
    ++i;
  }
}
// The wave's rows of the state as planes, where the team reads them.
template <int OWN>
__device__ static inline void put_state(const f32x4 (&S)[OWN], int own) {
  if constexpr (OWN > 1) {
#pragma unroll
    for (int s = 0; s < OWN / 2; ++s) {
      const Planes<3> f = split<3>(S[2 * s], S[2 * s + 1]);
#pragma unroll
      for (int p = 0; p < 3; ++p) lds_put(own + 1024 * (3 * s + p), f.p[p]);
    }
  } else {
    put_half<3>(own, split_half<3>(S[0]));
  }
}
// The wave's tiles of the state + K^T (Q^T) u: all steps' smallest terms first, or one step's products behind the other's (STEP).
template <typename L, int N>
__device__ static inline void mma_update(const Planes<L::NI> (&k)[N][L::NS], const Planes<3> (&u)[L::NS], f32x4 (&S)[N]) {
#pragma unroll
  for (int w = 2; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < L::NI; ++i)
      if (w - i >= 0)
#pragma unroll
        for (int s = 0; s < L::NS; ++s)
#pragma unroll
          for (int kt = 0; kt < N; ++kt) S[kt] = mma1(k[kt][s].p[i], u[s].p[w - i], S[kt]);
}
template <typename L, int N>
__device__ static inline void mma_update_step(const Planes<L::NI> (&k)[N][L::NS], const Planes<3> (&u)[L::NS], int s, f32x4 (&S)[N]) {
#pragma unroll
  for (int w = 2; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < L::NI; ++i)
      if (w - i >= 0)
#pragma unroll
        for (int kt = 0; kt < N; ++kt) S[kt] = mma1(k[kt][s].p[i], u[s].p[w - i], S[kt]);
}

template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC, bool FWD>
__device__ static __forceinline__ void team_scan(const Args& A) {
  constexpr int NO = Kind<T>::kOut, NP = FWD ? NO : 0;
  typedef TeamChunks<T, D1, TEAMS, NP, false, DIRECT> L;
  constexpr int C = L::C, KS = L::KS, NS = L::NS, NB = L::NB, NI = L::NI, OWN = L::kOwn, TEAM = L::kTeam;
  typedef typename L::MK MK;
  typedef typename L::MV MV;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, team = wave / TEAM, h = wave % TEAM;
  const int bh = blockIdx.x, col0 = blockIdx.y * L::VC, n = length_of(A, bh), c0 = col0 + 16 * team, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  const Rows xo = rows_at<T>(A.out, A, bh, A.dv, n, col0, min(A.dv - col0, L::VC));
  if (FWD && n < A.L) zero_rows<T>(xo, n, A.L, tid, L::kThreads);
  if (wave >= TEAM * TEAMS) {
    if (chunks > 0) load_team<L, D1, NP, VEC, false>(A, bh, A.V, col0, n, tid - 64 * TEAM * TEAMS);
    return;
  }
  f32x4 S[OWN];
#pragma unroll
  for (int kt = 0; kt < OWN; ++kt) S[kt] = zero4();
  if (A.s_in != nullptr) load_state<OWN, true>(S, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g, h * 16 * OWN);
  const TeamBases<L, false> base(l, lane, team, h);
  const bool two = NS == 2 && h >= 2;   // blocks of the wave's row tile
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tq = buf * L::kQ, tv = buf * L::kV, tt = buf * L::kT, tp = L::ps == 2 ? buf * L::kP : 0, tw = buf * L::kW;
    const int r0 = c * C, nr = min(C, n - r0);
    put_state(S, base.own);
    if (!FWD) {
      const Buffer to = buffer(A.states + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), (unsigned)(D1 * A.dvp) * 4u);
#pragma unroll
      for (int kt = 0; kt < OWN; ++kt) put_tile(S[kt], to, h * 16 * OWN + 16 * kt, A.dvp, c0, l);
    }
    Planes<NI> k[KS], q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      k[s] = MK::row(tk, base.rows, 0, s);
      if (FWD) q[s] = MK::row(tq, base.query, 0, s);
    }
    const f32x4 gamma = lds_get<f32x4>(base.vec + tw), left = lds_get<f32x4>(base.vec + tw + 4 * C), beta = lds_get<f32x4>(base.vec + tw + 4 * 2 * C);
    const f32x4 V = column<MV, NI>(base.value + tv);
    lds_barrier();
    Planes<3> b[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) b[s] = get_planes<3>(base.planes + 3 * 1024 * s);
    const f32x4 R = mma_steps<!DIRECT, NI, 3>(k, b, zero4());
    put_half<3>(base.half + L::x2 + (h >> 1) * 3 * 1024, split_half<3>(beta * (V - gamma * R)));
    Planes<3> t[2] = {get_block<NB, 3>(base.tri + tt)};
    if (NS == 2) t[1] = get_block<NB, 3>(base.tri + tt + (two ? 1024 : 0));
    f32x4 O = zero4(), U = zero4();
    lds_barrier();
    {
      const Planes<3> r = get_planes<3>(base.planes + L::x2);
      if (FWD) O = mma_steps<!DIRECT, NO, NI>(b, q, O);   // while the reads are on their way
      if (!DIRECT) U = mma_block<true, false>(t[0], r, U);
      if (two) U = mma_block<!DIRECT, false>(t[1], get_planes<3>(base.planes + L::x2 + 3 * 1024), U);
      if (DIRECT) U = mma_block<false, false>(t[0], r, U);
    }
    put_half<3>(base.half + (h >> 1) * 3 * 1024, split_half<3>(left * U));
    if (FWD) put_half<NO>(base.half + L::kRows + (h >> 1) * NO * 1024, split_half<NO>(U));
    const float Gamma = lds_get<float>(base.vec + tw + 4 * 3 * C);
    Planes<NI> kc[OWN][NS];
#pragma unroll
    for (int kt = 0; kt < OWN; ++kt) {
      S[kt] *= Gamma;
#pragma unroll
      for (int s = 0; s < NS; ++s) kc[kt][s] = MK::col(tk, base.cols, kt, s);
    }
    lds_barrier();
    {
      Planes<3> u[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) u[s] = get_planes<3>(base.planes + 3 * 1024 * s);
      if constexpr (DIRECT) {
        mma_update<L>(kc, u, S);
      } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) mma_update_step<L>(kc, u, s, S);
      }
    }
    if (FWD) {
      const Planes<NO> p0 = get_block<NB, NO>(base.weights + tp), u0 = get_planes<NO>(base.planes + L::kRows);
      O *= lds_get<float>(base.row + tw);
      if (!DIRECT) O = mma_block<true, true>(p0, u0, O);
      if (two) O = mma_block<!DIRECT, true>(get_block<NB, NO>(base.weights + tp + 1024), get_planes<NO>(base.planes + L::kRows + NO * 1024), O);
      if (DIRECT) O = mma_block<false, true>(p0, u0, O);
      const int row = 16 * h + l.i;
      const unsigned col = (unsigned)((16 * team + 4 * l.g) * (int)sizeof(T));
      if (VEC) buffer_quad<T>(xo.rows(r0, nr), row < nr && (DIRECT || col < xo.width) ? (unsigned)row * xo.row + col : kNowhere, A.scale * O);
      else if (row < nr && col < xo.width) store_quad<T>(xo.at(r0 + row) + col, (int)(xo.width - col), A.scale * O);
    } else {
      put_tile(U, buffer(A.u + chunk_at(A, bh, c) * ((long long)C * A.dvp), (unsigned)(C * A.dvp) * 4u), 16 * h, A.dvp, c0, l);
    }
    lds_barrier();
  };
  if (chunks > 0) each_chunk_of_team<false>(chunks, step);
  if (A.s_out != nullptr) store_state<OWN>(S, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g, h * 16 * OWN);
}

template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC>
__device__ static __forceinline__ void team_rev(const Args& A) {
  typedef TeamChunks<T, D1, TEAMS, 3, true, DIRECT> L;
  constexpr int C = L::C, KS = L::KS, NS = L::NS, NB = L::NB, NI = L::NI, OWN = L::kOwn, TEAM = L::kTeam;
  typedef typename L::MK MK;
  typedef typename L::MV MV;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, team = wave / TEAM, h = wave % TEAM;
  const int bh = blockIdx.x, col0 = blockIdx.y * L::VC, n = length_of(A, bh), c0 = col0 + 16 * team, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  if (wave >= TEAM * TEAMS) {
    if (chunks > 0) load_team<L, D1, 3, VEC, true>(A, bh, A.dOut, col0, n, tid - 64 * TEAM * TEAMS);
    return;
  }
  f32x4 G[OWN];
#pragma unroll
  for (int kt = 0; kt < OWN; ++kt) G[kt] = zero4();
  if (A.s_in != nullptr) load_state<OWN, true>(G, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g, h * 16 * OWN);
  const TeamBases<L, true> base(l, lane, team, h);
  const bool two = NS == 2 && h < 2;
  int vc = (MV::col_base(l) ^ (team << 5)) + L::v;
  asm("" : "+v"(vc));
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tq = L::qs == 2 ? buf * L::kQ : 0, tv = buf * L::kV, tt = L::ts == 2 ? buf * L::kT : 0, tp = buf * L::kP, tw = buf * L::kW;
    put_state(G, base.own);
    {
      const Buffer to = buffer(A.dstates + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), (unsigned)(D1 * A.dvp) * 4u);
#pragma unroll
      for (int kt = 0; kt < OWN; ++kt) put_tile(G[kt], to, h * 16 * OWN + 16 * kt, A.dvp, c0, l);
    }
    Planes<NI> k[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) k[s] = MK::row(tk, base.rows, 0, s);
    const f32x4 gamma = lds_get<f32x4>(base.vec + tw), left = lds_get<f32x4>(base.vec + tw + 4 * C), beta = lds_get<f32x4>(base.vec + tw + 4 * 2 * C);
    lds_barrier();
    Planes<3> b[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) b[s] = get_planes<3>(base.planes + 3 * 1024 * s);
    f32x4 D = zero4();   // scale P^T dO, while the reads are on their way
    {
      const Planes<3> p1 = get_block<NB, 3>(base.weights + tp);
      const Planes<NI> o1 = MV::col(tv, vc, 0, NS - 1);
      if (two) D = mma_block<!DIRECT, false>(get_block<NB, 3>(base.weights + tp - 1024), MV::col(tv, vc, 0, 0), D);
      if (DIRECT) D = mma_block<false, false>(p1, o1, D);
      else D += mma_block<true, false>(p1, o1, zero4());
    }
    const f32x4 U = mma_steps<!DIRECT, NI, 3>(k, b, zero4());
    put_half<3>(base.half + L::x2 + (h >> 1) * 3 * 1024, split_half<3>(left * U + D));
    const Half<3> o = split_half<3>(A.scale * gamma * column<MV, NI>(base.value + tv));
    lds_barrier();
    f32x4 R = zero4();
    {
      const Planes<3> t1 = get_block<NB, 3>(base.tri + tt), r1 = get_planes<3>(base.planes + L::x2 + (NS - 1) * 3 * 1024);
      if (two) R = mma_block<!DIRECT, false>(get_block<NB, 3>(base.tri + tt - 1024), get_planes<3>(base.planes + L::x2), R);
      if (DIRECT) R = mma_block<false, false>(t1, r1, R);
      else R += mma_block<true, false>(t1, r1, zero4());
    }
    put_half<3>(base.half + (h >> 1) * 3 * 1024, split_half<3>(-(gamma * beta) * R));
    put_half<3>(base.half + L::kRows + (h >> 1) * 3 * 1024, o);
    const float Gamma = lds_get<float>(base.vec + tw + 4 * 3 * C);
    Planes<NI> kc[OWN][NS];
#pragma unroll
    for (int kt = 0; kt < OWN; ++kt) {
      G[kt] *= Gamma;
#pragma unroll
      for (int s = 0; s < NS; ++s) kc[kt][s] = MK::col(tk, base.cols, kt, s);
    }
    lds_barrier();
    {
      Planes<3> u[NS], w[NS];
      Planes<NI> qc[OWN][NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        u[s] = get_planes<3>(base.planes + 3 * 1024 * s);
        w[s] = get_planes<3>(base.planes + L::kRows + 3 * 1024 * s);
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) qc[kt][s] = MK::col(tq, base.query_cols, kt, s);
      }
      if constexpr (DIRECT) {
        mma_update<L>(qc, w, G);
        mma_update<L>(kc, u, G);
      } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          mma_update_step<L>(qc, w, s, G);
          mma_update_step<L>(kc, u, s, G);
        }
      }
    }
    put_tile(R, buffer(A.dr + chunk_at(A, bh, c) * ((long long)C * A.dvp), (unsigned)(C * A.dvp) * 4u), 16 * h, A.dvp, c0, l);
    lds_barrier();
  };
  if (chunks > 0) each_chunk_of_team<true>(chunks, step);
  if (A.s_out != nullptr) store_state<OWN>(G, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g, h * 16 * OWN);
}

template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC>
__global__ __launch_bounds__((TeamChunks<T, D1, TEAMS, 3, true, DIRECT>::kThreads)) void k_delta_team(Args A) {
  team_scan<T, D1, TEAMS, DIRECT, VEC, true>(A);
}
// Backward: the gradients of the states (z = 0) and the states (z = 1) do not wait for each other.
template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC>
__global__ __launch_bounds__((TeamChunks<T, D1, TEAMS, 3, true, DIRECT>::kThreads)) void k_delta_team_back(Args A, const float* g_in, float* g_out) {
  if (blockIdx.z == 0) {
    A.s_in = g_in;
    A.s_out = g_out;
    team_rev<T, D1, TEAMS, DIRECT, VEC>(A);
  } else {
    team_scan<T, D1, TEAMS, DIRECT, VEC, false>(A);
  }
}

// Whether a call takes these kernels: DIRECT always; what goes through registers while each team of the launch has a CU to itself (48 heads of 1000 x 96 and
// 80, 240 teams: 42 us, one wave for 16 columns 55; fp32, 48 heads of 1000 x 64 backward, 384 teams: 95, one wave 75).
constexpr int kCUs = 256;
static long long teams_of(const Args& a, int cols) { return (long long)a.B * a.H * ((cols + 15) / 16); }
template <typename T>
static bool direct(const Args& a) { return sizeof(T) == 2 && (a.dk == 64 || a.dk == 128) && a.dv % 64 == 0; }
template <typename T>
static bool teamed(const Args& a) { return direct<T>(a) || (a.dk <= 128 && teams_of(a, a.dv) <= kCUs); }
template <typename T>
static bool teamed_back(const Args& a, bool states) { return direct<T>(a) || (a.dk <= 128 && teams_of(a, a.dvp) * (states ? 2 : 1) <= kCUs); }

// One team a workgroup as long as each of those has a CU to itself: the reads of LDS, 128 bytes a cycle, are what two share (24 x 4096 x 64 with
// one and two: 92 and 116 us, backward 102 and 122; 64 x 8192 x 128, 512 teams: 521 and 364).
template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC>
static dark_status go_team(const Args& a, hipStream_t st) {
  typedef TeamChunks<T, D1, TEAMS, Kind<T>::kOut, false, DIRECT> L;
  DARK_TRY(allow_lds(k_delta_team<T, D1, TEAMS, DIRECT, VEC>, L::all));
  DARK_LAUNCH(KID_DELTA_SCAN, st, (k_delta_team<T, D1, TEAMS, DIRECT, VEC>), dim3(a.B * a.H, (a.dv + L::VC - 1) / L::VC), dim3(L::kThreads), L::all, a);
  return DARK_OK;
}
template <typename T, int D1, int TEAMS, bool DIRECT, bool VEC>
static dark_status go_team_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  typedef TeamChunks<T, D1, TEAMS, 3, true, DIRECT> L;
  constexpr int more = TeamChunks<T, D1, TEAMS, 0, false, DIRECT>::all, lds = L::all > more ? L::all : more;
  DARK_TRY(allow_lds(k_delta_team_back<T, D1, TEAMS, DIRECT, VEC>, lds));
  DARK_LAUNCH(KID_DELTA_BACK, st, (k_delta_team_back<T, D1, TEAMS, DIRECT, VEC>), dim3(a.B * a.H, a.dvp / L::VC, states ? 2 : 1), dim3(L::kThreads), lds, a, g_in, g_out);
  return DARK_OK;
}
template <typename T, int D1>
static dark_status go_team(const Args& a, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (direct<T>(a)) return teams_of(a, a.dv) > kCUs ? go_team<T, D1, 2, true, true>(a, st) : go_team<T, D1, 1, true, true>(a, st);
  return vec_of<T>(a) ? go_team<T, D1, 1, false, true>(a, st) : go_team<T, D1, 1, false, false>(a, st);
}
template <typename T, int D1>
static dark_status go_team_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (direct<T>(a))
      return teams_of(a, a.dv) * (states ? 2 : 1) > kCUs ? go_team_back<T, D1, 2, true, true>(a, g_in, g_out, states, st) : go_team_back<T, D1, 1, true, true>(a, g_in, g_out, states, st);
  return vec_of<T>(a) ? go_team_back<T, D1, 1, false, true>(a, g_in, g_out, states, st) : go_team_back<T, D1, 1, false, false>(a, g_in, g_out, states, st);
}
template <typename T>
static dark_status launch_team(const Args& a, hipStream_t st) { return a.dk <= 64 ? go_team<T, 64>(a, st) : go_team<T, 128>(a, st); }
template <typename T>
static dark_status launch_team_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  return a.dk <= 64 ? go_team_back<T, 64>(a, g_in, g_out, states, st) : go_team_back<T, 128>(a, g_in, g_out, states, st);
}

}  // namespace delta
}  // namespace dark
