// The gated delta rule's scans with four waves for 16 columns of the state: bf16 rows that fill the tiles (see delta_scan.h for those of one wave).
//
// A wave takes an instruction in seven to twelve cycles, whatever it is, where the chunks' states hang on each other; what a SIMD does in that
// time grows with its waves.  So the 16 columns' work is dealt to four waves: each has one of the chunk's row tiles and a quarter of the
// state's rows.  What a wave has as sums and all four need as an operand goes through
// LDS: the state's planes, R, and U, with a barrier behind each.  Two waves bring the operands, a part between two barriers: the loads of a whole
// chunk at once keep their wave from the first barrier for as long as a third of the chunk takes.
// (One wave and four: prompt of 16 x 777 x 128 42 -> 27 us, prefill of 64 x 8192 x 128 415 -> 322, 24 x 4096 x 64 as training runs it 122 -> 78 and
// backward 160 -> 100; two waves with all loads at once were no faster than one.)
#pragma once

#include "delta_scan.h"

namespace dark {
namespace delta {

constexpr int kTeam = 4, kTeamLoaders = 2;   // waves of a team, and waves that load

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

// Operands in LDS: K, V (dO), vectors and one triangle for two chunks; what is needed late in a chunk for one: P forward, Q and T backward.
template <int D1, int TEAMS, int NP, bool REV>
struct TeamChunks {
  static constexpr int C = 64, NB = 6, VC = 16 * TEAMS, KS = D1 / 32, kThreads = 64 * (kTeam * TEAMS + kTeamLoaders);
  typedef Mat<C, D1, 1> MK;
  typedef Mat<C, VC, 1> MV;
  static constexpr int kQ = NP > 0 ? MK::kAll : 0, kV = MV::kAll, kW = kScanVecs * C * 4, kT = 3 * NB * 1024, kP = NP * NB * 1024;
  static constexpr int qs = REV ? 1 : 2, ts = REV ? 1 : 2, ps = REV ? 2 : 1;   // buffers
  static constexpr int k = 0, q = 2 * MK::kAll, v = q + qs * kQ, w = v + 2 * kV, t = w + 2 * kW, p = t + ts * kT, x = p + ps * kP;
  // exchange, of a team: the state's planes, in their place later U's (those of the update, and those of P U or of dO); R's
  static constexpr int kMore = REV ? 6 * 1024 : 2 * NP * 1024;
  static constexpr int kFirst = KS * 3 * 1024, kLast = 6 * 1024 + kMore, x1 = 0, x2 = kFirst > kLast ? kFirst : kLast, kX = x2 + 6 * 1024;
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
      "s_mov_b32 m0, %5\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %4 offset:1024\n\t"
      "global_load_lds_dwordx4 %2, %4 offset:2048\n\tglobal_load_lds_dwordx4 %3, %4 offset:3072" ::"v"(off[0]),
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

// A lane's bases: those of row tile h, and of the wave's quarter of the state's rows.
template <typename L, bool REV>
struct TeamBases {
  static constexpr int RB = L::MK::RB, RV = L::MV::RB, kOwn = RB / 128;   // column tiles of K that are the wave's rows of the state
  int rows, cols, value, vec, row, tri, weights, planes, own, half;
  __device__ TeamBases(Lane l, int lane, int team, int h) {
    rows = L::MK::row_base(l) + h * 16 * RB;
    cols = L::MK::col_base(l) ^ (h * kOwn << 5);
    value = (L::MV::col_base(l) ^ (team << 5)) + h * 16 * RV + L::v;
    vec = 16 * l.g + L::w + 64 * h;
    row = 4 * l.i + L::w + 64 * h;
    // a lower triangle's row tile has block (h, 0), and (h, 1) behind it; of an upper one (h, 1), and (h, 0) before it
    const int first = REV ? (h < 2 ? 2 * h + 1 : h + 2) : h < 2 ? h : 2 * h - 2;
    tri = 16 * lane + L::t + 1024 * first;
    weights = 16 * lane + L::p + 1024 * first;
    planes = 16 * lane + L::x + team * L::kX;
    own = planes + (kOwn == 2 ? h * 3 * 1024 : (h >> 1) * 3 * 1024 + 8 * (h & 1));
    half = planes + 8 * (h & 1);
#pragma unroll
    for (int* p : {&rows, &cols, &value, &vec, &row, &tri, &weights, &planes, &own, &half}) asm("" : "+v"(*p));
  }
};

// Inner values 32 s ... of a row at a base of its own.
__device__ static inline u32x4 row_at(int base, int s) {
  const int at = base ^ (s << 6);
  const u32x2 a = lds_get<u32x2>(at), b = lds_get<u32x2>(at ^ 32);
  return u32x4{a[0], a[1], b[0], b[1]};
}
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
template <int M>
__device__ static inline void get_block(u32x4 (&t)[M], int at) {
#pragma unroll
  for (int i = 0; i < M; ++i) t[i] = lds_get<u32x4>(at + i * 6 * 1024);
}
// The four values of a tile's column from two words of bf16.
__device__ static inline f32x4 widen(u32x2 v) {
  return f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
}
// A tile's column to scratch.
__device__ static inline void put_tile(f32x4 v, Buffer b, int row, int stride, int c0, Lane l) {
  const unsigned at = (unsigned)((row + 4 * l.g) * stride + c0 + l.i) * 4u;
#pragma unroll
  for (int j = 0; j < 4; ++j) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[j]), b, at, (unsigned)(j * stride) * 4u, 0);
}
// x + t b for one block of a triangle in M planes (TRANS: b t).
template <int M, int N, bool TRANS>
__device__ static inline f32x4 mma_block(const u32x4 (&t)[M], const Planes<N>& b, f32x4 x) {
  constexpr int W = M > N ? M : N;
#pragma unroll
  for (int w = W - 1; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (w - i >= 0 && w - i < N) x = TRANS ? mma1(b.p[w - i], t[i], x) : mma1(t[i], b.p[w - i], x);
  return x;
}
// The wave's rows of the state as planes, where the team reads them.
template <int OWN>
__device__ static inline void put_state(const f32x4 (&S)[OWN], int own) {
  if constexpr (OWN == 2) {
    const Planes<3> f = split<3>(S[0], S[1]);
#pragma unroll
    for (int p = 0; p < 3; ++p) lds_put(own + 1024 * p, f.p[p]);
  } else {
    put_half<3>(own, split_half<3>(S[0]));
  }
}

template <int D1, int TEAMS, bool FWD>
__global__ __launch_bounds__((TeamChunks<D1, TEAMS, (FWD ? 2 : 0), false>::kThreads)) void k_delta_team(Args A) {
  constexpr int NO = 2, NP = FWD ? NO : 0;
  typedef TeamChunks<D1, TEAMS, NP, false> L;
  constexpr int C = L::C, KS = D1 / 32, OWN = D1 / 64;
  typedef typename L::MK MK;
  typedef unsigned short T;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, team = wave / kTeam, h = wave % kTeam;
  const int bh = blockIdx.x, col0 = blockIdx.y * L::VC, n = length_of(A, bh), c0 = col0 + 16 * team, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  const Rows xo = rows_at<T>(A.out, A, bh, A.dv, n, col0, L::VC);
  if (FWD && n < A.L) zero_rows<T>(xo, n, A.L, tid, L::kThreads);
  if (wave >= kTeam * TEAMS) {
    if (chunks == 0) return;
    if (wave == kTeam * TEAMS) load_keys<L, D1, NP, false>(A, bh, n, lane);
    else load_rest<L, D1, NP, false>(A, bh, rows_at<T>(A.V, A, bh, A.dv, n, col0, L::VC), n, lane);
    return;
  }
  f32x4 S[OWN];
#pragma unroll
  for (int kt = 0; kt < OWN; ++kt) S[kt] = zero4();
  if (A.s_in != nullptr) load_state<OWN, true>(S, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g, h * (D1 / 4));
  const TeamBases<L, false> base(l, lane, team, h);
  const bool two = h >= 2;   // blocks of the wave's row tile
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tq = L::q + buf * L::kQ, tv = buf * L::kV, tt = buf * L::kT, tw = buf * L::kW;
    const int r0 = c * C, nr = min(C, n - r0);
    put_state(S, base.own);
    if (!FWD) {
      const Buffer to = buffer(A.states + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), (unsigned)(D1 * A.dvp) * 4u);
#pragma unroll
      for (int kt = 0; kt < OWN; ++kt) put_tile(S[kt], to, h * (D1 / 4) + 16 * kt, A.dvp, c0, l);
    }
    u32x4 k[KS], q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      k[s] = row_at(base.rows + tk, s);
      if (FWD) q[s] = row_at(base.rows + tq, s);
    }
    const f32x4 gamma = lds_get<f32x4>(base.vec + tw), left = lds_get<f32x4>(base.vec + tw + 4 * C), beta = lds_get<f32x4>(base.vec + tw + 4 * 2 * C);
    const f32x4 V = widen(lds_get_tr16(base.value + tv));
    lds_barrier();
    Planes<3> b[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) b[s] = get_planes<3>(base.planes + 3 * 1024 * s);
    f32x4 R = zero4(), O = zero4(), U = zero4();
#pragma unroll
    for (int i = 2; i >= 0; --i)
#pragma unroll
      for (int s = 0; s < KS; ++s) R = mma1(k[s], b[s].p[i], R);
    put_half<3>(base.half + L::x2 + (h >> 1) * 3 * 1024, split_half<3>(beta * (V - gamma * R)));
    u32x4 t0[3], t1[3];
    get_block<3>(t0, base.tri + tt);
    get_block<3>(t1, base.tri + tt + (two ? 1024 : 0));
    if (FWD) {
#pragma unroll
      for (int i = NO - 1; i >= 0; --i)
#pragma unroll
        for (int s = 0; s < KS; ++s) O = mma1(b[s].p[i], q[s], O);
    }
    lds_barrier();
    {
      const Planes<3> r0 = get_planes<3>(base.planes + L::x2);
      if (two) {
        const Planes<3> r1 = get_planes<3>(base.planes + L::x2 + 3 * 1024);
        U = mma_block<3, 3, false>(t1, r1, U);
      }
      U = mma_block<3, 3, false>(t0, r0, U);
    }
    put_half<3>(base.half + (h >> 1) * 3 * 1024, split_half<3>(left * U));
    if (FWD) put_half<NO>(base.half + 6 * 1024 + (h >> 1) * NO * 1024, split_half<NO>(U));
    const float Gamma = lds_get<float>(base.vec + tw + 4 * 3 * C);
    u32x4 kt0[OWN], kt1[OWN];
#pragma unroll
    for (int kt = 0; kt < OWN; ++kt) {
      S[kt] *= Gamma;
      kt0[kt] = MK::col(tk, base.cols, kt, 0).p[0];
      kt1[kt] = MK::col(tk, base.cols, kt, 1).p[0];
    }
    lds_barrier();
    {
      const Planes<3> u0 = get_planes<3>(base.planes), u1 = get_planes<3>(base.planes + 3 * 1024);
#pragma unroll
      for (int i = 2; i >= 0; --i) {
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) S[kt] = mma1(kt0[kt], u0.p[i], S[kt]);
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) S[kt] = mma1(kt1[kt], u1.p[i], S[kt]);
      }
    }
    if (FWD) {
      u32x4 p0[NO];
      get_block<NO>(p0, base.weights);
      O *= lds_get<float>(base.row + tw);
      if (two) {
        u32x4 p1[NO];
        get_block<NO>(p1, base.weights + 1024);
        O = mma_block<NO, NO, true>(p1, get_planes<NO>(base.planes + 6 * 1024 + NO * 1024), O);
      }
      O = mma_block<NO, NO, true>(p0, get_planes<NO>(base.planes + 6 * 1024), O);
      const int row = 16 * h + l.i;
      buffer_quad<T>(xo.rows(r0, nr), row < nr ? (unsigned)row * xo.row + (unsigned)((16 * team + 4 * l.g) * (int)sizeof(T)) : kNowhere, A.scale * O);
    } else {
      put_tile(U, buffer(A.u + chunk_at(A, bh, c) * ((long long)C * A.dvp), (unsigned)(C * A.dvp) * 4u), 16 * h, A.dvp, c0, l);
    }
    lds_barrier();
  };
  if (chunks > 0) {
    lds_barrier();
    for (int i = 0; i < chunks;) {
      step(i, std::integral_constant<int, 0>());
      if (++i == chunks) break;
      step(i, std::integral_constant<int, 1>());
      ++i;
    }
  }
  if (A.s_out != nullptr) store_state<OWN>(S, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g, h * (D1 / 4));
}

template <int D1, int TEAMS>
__global__ __launch_bounds__((TeamChunks<D1, TEAMS, 3, true>::kThreads)) void k_delta_team_rev(Args A) {
  typedef TeamChunks<D1, TEAMS, 3, true> L;
  constexpr int C = L::C, KS = D1 / 32, OWN = D1 / 64;
  typedef typename L::MK MK;
  typedef typename L::MV MV;
  typedef unsigned short T;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, team = wave / kTeam, h = wave % kTeam;
  const int bh = blockIdx.x, col0 = blockIdx.y * L::VC, n = length_of(A, bh), c0 = col0 + 16 * team, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  if (wave >= kTeam * TEAMS) {
    if (chunks == 0) return;
    if (wave == kTeam * TEAMS) load_keys<L, D1, 3, true>(A, bh, n, lane);
    else load_rest<L, D1, 3, true>(A, bh, rows_at<T>(A.dOut, A, bh, A.dv, n, col0, L::VC), n, lane);
    return;
  }
  f32x4 G[OWN];
#pragma unroll
  for (int kt = 0; kt < OWN; ++kt) G[kt] = zero4();
  if (A.s_in != nullptr) load_state<OWN, true>(G, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g, h * (D1 / 4));
  const TeamBases<L, true> base(l, lane, team, h);
  const bool two = h < 2;
  int vc = (MV::col_base(l) ^ (team << 5)) + L::v;
  asm("" : "+v"(vc));
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tv = buf * L::kV, tp = buf * L::kP, tw = buf * L::kW;
    put_state(G, base.own);
    {
      const Buffer to = buffer(A.dstates + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), (unsigned)(D1 * A.dvp) * 4u);
#pragma unroll
      for (int kt = 0; kt < OWN; ++kt) put_tile(G[kt], to, h * (D1 / 4) + 16 * kt, A.dvp, c0, l);
    }
    u32x4 k[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) k[s] = row_at(base.rows + tk, s);
    const f32x4 gamma = lds_get<f32x4>(base.vec + tw), left = lds_get<f32x4>(base.vec + tw + 4 * C), beta = lds_get<f32x4>(base.vec + tw + 4 * 2 * C);
    f32x4 U = zero4(), R = zero4(), D = zero4();
    {
      u32x4 p1[3];
      get_block<3>(p1, base.weights + tp);
      const u32x4 o1 = MV::col(tv, vc, 0, 1).p[0];
#pragma unroll
      for (int i = 2; i >= 0; --i) D = mma1(p1[i], o1, D);
      if (two) {
        u32x4 p0[3];
        get_block<3>(p0, base.weights + tp - 1024);
        const u32x4 o0 = MV::col(tv, vc, 0, 0).p[0];
#pragma unroll
        for (int i = 2; i >= 0; --i) D = mma1(p0[i], o0, D);
      }
    }
    lds_barrier();
    Planes<3> b[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) b[s] = get_planes<3>(base.planes + 3 * 1024 * s);
#pragma unroll
    for (int i = 2; i >= 0; --i)
#pragma unroll
      for (int s = 0; s < KS; ++s) U = mma1(k[s], b[s].p[i], U);
    put_half<3>(base.half + L::x2 + (h >> 1) * 3 * 1024, split_half<3>(left * U + D));
    const Half<3> o = split_half<3>(A.scale * gamma * widen(lds_get_tr16(base.value + tv)));
    lds_barrier();
    {
      u32x4 t1[3];
      get_block<3>(t1, base.tri);
      const Planes<3> r1 = get_planes<3>(base.planes + L::x2 + 3 * 1024);
      if (two) {
        u32x4 t0[3];
        get_block<3>(t0, base.tri - 1024);
        R = mma_block<3, 3, false>(t0, get_planes<3>(base.planes + L::x2), R);
      }
      R = mma_block<3, 3, false>(t1, r1, R);
    }
    put_half<3>(base.half + (h >> 1) * 3 * 1024, split_half<3>(-(gamma * beta) * R));
    put_half<3>(base.half + 6 * 1024 + (h >> 1) * 3 * 1024, o);
    const float Gamma = lds_get<float>(base.vec + tw + 4 * 3 * C);
    u32x4 kt0[OWN], kt1[OWN];
#pragma unroll
    for (int kt = 0; kt < OWN; ++kt) {
      G[kt] *= Gamma;
      kt0[kt] = MK::col(tk, base.cols, kt, 0).p[0];
      kt1[kt] = MK::col(tk, base.cols, kt, 1).p[0];
    }
    lds_barrier();
    {
      const Planes<3> u0 = get_planes<3>(base.planes), u1 = get_planes<3>(base.planes + 3 * 1024);
      const Planes<3> o0 = get_planes<3>(base.planes + 6 * 1024), o1 = get_planes<3>(base.planes + 9 * 1024);
      u32x4 q0[OWN], q1[OWN];
#pragma unroll
      for (int kt = 0; kt < OWN; ++kt) {
        q0[kt] = MK::col(L::q, base.cols, kt, 0).p[0];
        q1[kt] = MK::col(L::q, base.cols, kt, 1).p[0];
      }
#pragma unroll
      for (int i = 2; i >= 0; --i) {
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) G[kt] = mma1(kt0[kt], u0.p[i], G[kt]);
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) G[kt] = mma1(kt1[kt], u1.p[i], G[kt]);
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) G[kt] = mma1(q0[kt], o0.p[i], G[kt]);
#pragma unroll
        for (int kt = 0; kt < OWN; ++kt) G[kt] = mma1(q1[kt], o1.p[i], G[kt]);
      }
    }
    put_tile(R, buffer(A.dr + chunk_at(A, bh, c) * ((long long)C * A.dvp), (unsigned)(C * A.dvp) * 4u), 16 * h, A.dvp, c0, l);
    lds_barrier();
  };
  if (chunks > 0) {
    lds_barrier();
    for (int i = 0; i < chunks;) {
      step(chunks - 1 - i, std::integral_constant<int, 0>());
      if (++i == chunks) break;
      step(chunks - 1 - i, std::integral_constant<int, 1>());
      ++i;
    }
  }
  if (A.s_out != nullptr) store_state<OWN>(G, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g, h * (D1 / 4));
}

// Whether a call takes these kernels.
static bool teamed(const Args& a) { return (a.dk == 64 || a.dk == 128) && a.dv % 64 == 0; }

// One team a workgroup as long as each of those has a CU to itself: the reads of LDS, 128 bytes a cycle, are what two share (24 x 4096 x 64 with
// one and two: 78 and 98 us, backward 100 and 124).
constexpr int kCUs = 256;
template <int D1, int TEAMS, bool FWD>
static dark_status go_team(const Args& a, hipStream_t st) {
  typedef TeamChunks<D1, TEAMS, (FWD ? 2 : 0), false> L;
  DARK_TRY(allow_lds(k_delta_team<D1, TEAMS, FWD>, L::all));
  DARK_LAUNCH(KID_DELTA_SCAN, st, (k_delta_team<D1, TEAMS, FWD>), dim3(a.B * a.H, a.dv / L::VC), dim3(L::kThreads), L::all, a);
  return DARK_OK;
}
template <int D1, int TEAMS>
static dark_status go_team_rev(const Args& a, hipStream_t st) {
  typedef TeamChunks<D1, TEAMS, 3, true> L;
  DARK_TRY(allow_lds(k_delta_team_rev<D1, TEAMS>, L::all));
  DARK_LAUNCH(KID_DELTA_REV, st, (k_delta_team_rev<D1, TEAMS>), dim3(a.B * a.H, a.dv / L::VC), dim3(L::kThreads), L::all, a);
  return DARK_OK;
}
static bool one_team(const Args& a) { return (long long)a.B * a.H * (a.dv / 16) <= kCUs; }
template <int D1, bool FWD>
static dark_status go_team(const Args& a, hipStream_t st) { return one_team(a) ? go_team<D1, 1, FWD>(a, st) : go_team<D1, 2, FWD>(a, st); }
template <int D1>
static dark_status go_team_rev(const Args& a, hipStream_t st) { return one_team(a) ? go_team_rev<D1, 1>(a, st) : go_team_rev<D1, 2>(a, st); }

}  // namespace delta
}  // namespace dark
