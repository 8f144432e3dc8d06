// The gated delta rule chunk by chunk: the chunks' triangles, and the scans over them (see delta.h for the mathematics).
#pragma once

#include <type_traits>

#include "delta_tile.h"

namespace dark {
namespace delta {

// ---------------------------------------------------------------------------
// T = (I + diag(beta) E)^-1 and P = D o (Q K^T) of every chunk, in operand order; backward their transposes, P times scale.
// The inverse: blocks of 16 x 16 on the diagonal by substitution, row after row; below it T_rc = -T_rr sum_m A_rm T_mc, by fp32 matrix
// products, one diagonal of blocks after the other.  Substitution and products are backward stable for any beta and keys.
// A chunk a workgroup.  Many chunks are bound by memory: 8192 of 64 x 128 in bf16 take 104 to 115 us, 62 KB each (K and Q read, T in three planes and P in two
// written), 4.4 to 4.9 TB/s; 1536 of 64 x 64 22, backward, with T^T and a third plane of P, 27.  Few are bound by the steps one after the other: 208 take 10.
// ---------------------------------------------------------------------------
template <typename T, int D1>
constexpr int prep_lds() {
  constexpr int C = Kind<T>::kChunk;
  constexpr int tiles = 2 * Mat<C, D1, Kind<T>::kIn>::kAll, square = 4 * C * (C + 4);
  return (tiles >= square ? tiles : tiles + square) + square + kVecs * C * 4;   // T in the place of K and Q where it fits
}

template <typename T, int D1, bool VEC, bool BWD>
__global__ __launch_bounds__(256) void k_delta_prep(Args A) {
  constexpr int C = Kind<T>::kChunk, NT = C / 16, NI = Kind<T>::kIn, NB = blocks_of(C), NTH = 256, S = C + 4;
  typedef Mat<C, D1, NI> M;
  constexpr int tk = 0, tq = M::kAll, ta = 2 * M::kAll, tt = ta >= 4 * C * S ? 0 : ta + 4 * C * S, tv = tt == 0 ? ta + 4 * C * S : tt + 4 * C * S;
  constexpr int NP = BWD ? 3 : Kind<T>::kOut;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int bh = blockIdx.x / A.chunks, c = blockIdx.x % A.chunks, r0 = c * C, n = length_of(A, bh), nr = min(C, n - r0);
  if (nr <= 0) return;
  {
    const Rows k = rows_at<T>(A.K, A, bh, A.dk, n, 0, A.dk), q = rows_at<T>(A.Q, A, bh, A.dk, n, 0, A.dk);
    Load<T, C, D1, NTH, VEC> lk, lq;
    lk.load(k, r0, nr, tid);
    lq.load(q, r0, nr, tid);
    if (wave == 0) {
      // Sums of log gates in 64 bits, as two floats: their differences are as exact as the gates.  exp(-1e4) is 0; -infinity would
      // leave infinity - infinity.
      float g = 0.f, be = 0.f;
      if (lane < nr) {
        if (A.log_gate != nullptr) g = A.log_gate[gate_at(A, bh, r0 + lane)];
        be = A.beta[gate_at(A, bh, r0 + lane)];
        g = g < -1e4f ? -1e4f : g;
      }
      double G = (double)g;
#pragma unroll
      for (int o = 1; o < C; o <<= 1) {
        const double x = __shfl_up(G, o, 64);
        if (lane >= o) G += x;
      }
      const double end = __shfl(G, C - 1, 64);
      const float hi = (float)G, lo = (float)(G - (double)hi);
      if (lane < C) {
        const bool there = lane < nr;   // rows behind the last weigh nothing, whatever stands there
        const float v[kVecs] = {there ? expf((float)G) : 0.f, there ? expf((float)(end - G)) : 0.f, be, expf((float)end), hi, lo};
        float* const to = A.vec + chunk_at(A, bh, c) * (kVecs * C);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          lds_put(tv + 4 * (i * C + lane), v[i]);
          to[i * C + lane] = v[i];
        }
      }
    }
    lk.template store<M>(tk, tid);
    lq.template store<M>(tq, tid);
  }
  __syncthreads();
  const Lane l{lane & 15, lane >> 4};
  const int rb = M::row_base(l);
  const auto elem = [&](int base, int r, int col) { return base + 4 * (r * S + col); };
  const long long own = chunk_at(A, bh, c);
  // A block of P (P^T) as an operand takes two tiles, next to each other in its inner index: with that index along a lane's accumulators, they are
  // the operand as they come.  Lane index i of tile `row`, accumulators of the tiles of step s; forward rows are tokens t, backward keys i.
  const auto block = [&](int blk) {
    const int row = C == 32 ? blk : !BWD ? (blk < 2 ? blk : blk < 4 ? 2 : 3) : blk < 4 ? blk >> 1 : blk - 2;
    const int s = C == 32 ? 0 : !BWD ? (blk < 2 ? 0 : blk & 1) : blk < 4 ? blk & 1 : 1;
    const int own_at = 16 * row + l.i;
    const float hi = lds_get<float>(tv + 4 * (4 * C + own_at)), lo = lds_get<float>(tv + 4 * (5 * C + own_at));
    f32x4 P[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int in = 2 * s + h, qt = BWD ? in : row, kt = BWD ? row : in;
      P[h] = zero4();
      if (kt > qt) continue;
      f32x4 kk = zero4(), qk = zero4();
#pragma unroll
      for (int e = 0; e < D1 / 32; ++e) {
        const Planes<NI> k = M::row(tk, rb, kt, e), kq = M::row(tk, rb, qt, e), q = M::row(tq, rb, qt, e);
        kk = BWD ? mma(kq, k, kk) : mma(k, kq, kk);
        qk = BWD ? mma(q, k, qk) : mma(k, q, qk);
      }
      const f32x4 his = lds_get<f32x4>(tv + 4 * (4 * C + 16 * in + 4 * l.g)), los = lds_get<f32x4>(tv + 4 * (5 * C + 16 * in + 4 * l.g));
      const f32x4 bes = lds_get<f32x4>(tv + 4 * (2 * C + 16 * in + 4 * l.g));
      const float be = lds_get<float>(tv + 4 * (2 * C + own_at));
      f32x4 E;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int in_at = 16 * in + 4 * l.g + j, t = BWD ? in_at : own_at, i = BWD ? own_at : in_at;
        const float d = expf(BWD ? (his[j] - hi) + (los[j] - lo) : (hi - his[j]) + (lo - los[j]));
        P[h][j] = t >= i ? (BWD ? A.scale : 1.f) * d * qk[j] : 0.f;
        E[j] = t > i ? (BWD ? bes[j] : be) * d * kk[j] : 0.f;
        if (BWD) lds_put(elem(ta, t, i), E[j]);
      }
      if (!BWD) lds_put(elem(ta, own_at, 16 * in + 4 * l.g), E);
    }
    const Planes<NP> f = split<NP>(P[0], P[1]);
#pragma unroll
    for (int k = 0; k < NP; ++k) A.pri[(own * NP + k) * (NB * 64) + 64 * blk + lane] = f.p[k];
  };
  // blocks of one tile and of two: each wave two or three tiles
  if (C == 32) {
    if (wave < 2) block(wave);
  } else if (BWD) {
    block(wave == 0 ? 0 : wave == 1 ? 1 : wave == 2 ? 3 : 4);
    if (wave >= 2) block(wave == 2 ? 2 : 5);
  } else {
    block(wave == 0 ? 4 : wave == 1 ? 5 : wave == 2 ? 2 : 1);
    if (wave >= 2) block(wave == 2 ? 0 : 3);
  }
  __syncthreads();
  if (wave < NT) {
    // x: column l.i of the block's inverse, the same in every lane group
    float x[16];
    const int at = elem(ta, 16 * wave, 16 * wave);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float v = r == l.i ? 1.f : 0.f;
      f32x4 a = zero4();
#pragma unroll
      for (int i = 0; i < r; ++i) {
        if (i % 4 == 0) a = lds_get<f32x4>(at + 4 * (r * S + i));
        v -= a[i % 4] * x[i];
      }
      x[r] = v;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (r / 4 == l.g) lds_put(elem(tt, 16 * wave + r, 16 * wave + l.i), x[r]);
  }
#pragma unroll
  for (int d = 1; d < NT; ++d) {
    __syncthreads();
    const int cc = wave, rr = wave + d;
    if (rr < NT) {
      f32x4 y = zero4();
#pragma unroll
      for (int m = 0; m < d; ++m) {
        const f32x4 a = lds_get<f32x4>(elem(ta, 16 * rr + l.i, 16 * (cc + m) + 4 * l.g));
#pragma unroll
        for (int k = 0; k < 4; ++k)
          y = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], lds_get<float>(elem(tt, 16 * (cc + m) + 4 * l.g + k, 16 * cc + l.i)), y, 0, 0, 0);
      }
      const f32x4 a = lds_get<f32x4>(elem(tt, 16 * rr + l.i, 16 * rr + 4 * l.g));
      f32x4 z = zero4();
#pragma unroll
      for (int k = 0; k < 4; ++k) z = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], y[k], z, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) lds_put(elem(tt, 16 * rr + 4 * l.g + k, 16 * cc + l.i), -z[k]);
    }
  }
  __syncthreads();
  for (int u = tid; u < NB * 64; u += NTH) {
    const int blk = u >> 6, i = u & 15, g = u >> 4 & 3;
    {
      const int r = C == 32 || blk < 2 ? blk : blk < 4 ? 2 : 3, s = C == 32 || blk < 2 ? 0 : blk & 1;
      const int at = elem(tt, 16 * r + i, 32 * s + 4 * g);
      const Planes<3> t = split<3>(lds_get<f32x4>(at), 2 * s + 1 <= r ? lds_get<f32x4>(at + 64) : zero4());   // nothing stands above the diagonal
#pragma unroll
      for (int k = 0; k < 3; ++k) A.tri[(own * 3 + k) * (NB * 64) + u] = t.p[k];
    }
    if (BWD) {
      const int r = C == 32 ? blk : blk < 4 ? blk >> 1 : blk - 2, s = C == 32 ? 0 : blk < 4 ? blk & 1 : 1;
      f32x4 v[2] = {zero4(), zero4()};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = elem(tt, 32 * s + 4 * g + j, 16 * r + i);
        if (2 * s >= r) v[0][j] = lds_get<float>(at);
        v[1][j] = lds_get<float>(at + 64 * S);
      }
      const Planes<3> t = split<3>(v[0], v[1]);
#pragma unroll
      for (int k = 0; k < 3; ++k) A.trit[(own * 3 + k) * (NB * 64) + u] = t.p[k];
    }
  }
}

// ---------------------------------------------------------------------------
// Chunk after chunk.  A wave owns 16 columns of the state, in the accumulators of the products that update it, and takes them through
// all of a chunk's products by itself: its state is an operand of K S and Q S, R of T R, U of P U and of the update, all without a way
// through LDS or another wave.  Further waves bring the next chunk's operands to LDS meanwhile: a wave that has its SIMD to itself takes several
// cycles for an instruction, whatever it is, so that the chain from state to state is as long as it has instructions.
// (bf16, 64 heads of 8192 x 120 and 128: 418 us; 64 heads of 2048 x 256 and 128: 203; fp32, 96 heads of 1024 x 64: 69, backward 94.)
// ---------------------------------------------------------------------------
// A chunk's operands in LDS (NP: planes of P, 0: neither Q nor P), in one buffer or two.  An instruction's own offset reaches 64 KB: a lane has a
// base for each operand, and the buffers lie beside each other.
// Four waves take them there through registers (two beside 256 rows of a state).
template <typename T, int D1, int NW, int NP>
struct Chunks {
  static constexpr int C = Kind<T>::kChunk, NI = Kind<T>::kIn, NB = blocks_of(C), VC = 16 * NW;
  typedef Mat<C, D1, NI> MK;
  typedef Mat<C, VC, NI> MV;
  static constexpr int kV = MV::kAll, kW = kScanVecs * C * 4, kT = 3 * NB * 1024, kP = NP * NB * 1024, kQ = NP > 0 ? MK::kAll : 0;   // bytes of each
  static constexpr int kBufs = 2 * (MK::kAll + kQ + kV + kW + kT + kP) <= 160 * 1024 ? 2 : 1;
  static constexpr int k = 0, q = k + kBufs * MK::kAll, v = q + kBufs * kQ, w = v + kBufs * kV, t = w + kBufs * kW, p = t + kBufs * kT, all = p + kBufs * kP;
  static constexpr int kLoaders = D1 > 128 ? 2 : 4, kThreads = 64 * (NW + kLoaders), NTH = 64 * kLoaders;
};

// A lane's bases.  The compiler is not to take them apart: it would hold one for every read behind the first 64 KB.
template <typename L>
struct Bases {
  static constexpr bool kFar = L::q + L::kBufs * L::kQ > 65536;   // K and Q do not share bases
  int rows, query, cols, query_cols, value, tri, weights, vec, vec_row;
  __device__ Bases(Lane l, int lane, int wave)
      : rows(L::MK::row_base(l)), query(rows + (kFar ? L::q : 0)), cols(L::MK::col_base(l)), query_cols(cols + (kFar ? L::q : 0)),
        value((L::MV::col_base(l) ^ (wave << 5)) + L::v), tri(16 * lane + L::t), weights(16 * lane + L::p), vec(16 * l.g + L::w), vec_row(4 * l.i + L::w) {
    if (kFar) {
      asm("" : "+v"(query));
      asm("" : "+v"(query_cols));
    }
    asm("" : "+v"(value));
    asm("" : "+v"(tri));
    asm("" : "+v"(weights));
    asm("" : "+v"(vec));
    asm("" : "+v"(vec_row));
  }
};

// The loading waves: chunk after chunk (REV: from the last to the first), one ahead.
template <typename L, typename T, int D1, int NP, bool VEC, bool REV>
__device__ static inline void load_chunks(const Args& A, int bh, const Rows& xk, const Rows& xq, const Rows& xv, int n, int tid) {
  constexpr int C = L::C, NB = L::NB, NTH = L::NTH;
  const int chunks = (n + C - 1) / C;
  const auto chunk = [&](int i) { return REV ? chunks - 1 - i : i; };
  const u32x4* const tri = REV ? A.trit : A.tri;
  Load<T, C, D1, NTH, VEC> lk, lq;
  Load<T, C, L::VC, NTH, VEC> lv;
  LoadTri<NB, 3, NTH> lt;
  LoadTri<NB, (NP > 0 ? NP : 1), NTH> lp;
  f32x4 lw;
  const auto load = [&](int i) {
    const int c = chunk(i), r0 = c * C, nr = min(C, n - r0);
    const long long own = chunk_at(A, bh, c);
    lk.load(xk, r0, nr, tid);
    if (NP > 0) lq.load(xq, r0, nr, tid);
    lv.load(xv, r0, nr, tid);
    lt.load(tri + own * (3 * NB * 64), tid);
    if (NP > 0) lp.load(A.pri + own * (NP * NB * 64), tid);
    if (tid < C) lw = reinterpret_cast<const f32x4*>(A.vec + own * (kVecs * C))[tid];
  };
  const auto store = [&](int buf) {
    lk.template store<typename L::MK>(L::k + buf * L::MK::kAll, tid);
    if (NP > 0) lq.template store<typename L::MK>(L::q + buf * L::kQ, tid);
    lv.template store<typename L::MV>(L::v + buf * L::kV, tid);
    lt.store(L::t + buf * L::kT, tid);
    if (NP > 0) lp.store(L::p + buf * L::kP, tid);
    if (tid < C) lds_put(L::w + buf * L::kW + 16 * tid, lw);
  };
  load(0);
  store(0);
  if (chunks > 1) load(1);
  lds_barrier();
  for (int i = 0; i < chunks; ++i) {
    if (L::kBufs == 1) lds_barrier();   // the chunk's readers are done
    if (i + 1 < chunks) {
      store((i + 1) % L::kBufs);
      if (i + 2 < chunks) load(i + 2);
    }
    lds_barrier();
  }
}
// The computing waves: f(chunk, the buffer of its operands, a constant) for every chunk.
template <typename L, bool REV, typename F>
__device__ static inline void each_chunk(int chunks, const F& f) {
  lds_barrier();
  for (int i = 0; i < chunks;) {
    f(REV ? chunks - 1 - i : i, std::integral_constant<int, 0>());
    if (L::kBufs == 1) lds_barrier();
    lds_barrier();
    ++i;
    if (L::kBufs == 1 || i == chunks) continue;
    f(REV ? chunks - 1 - i : i, std::integral_constant<int, 1>());
    lds_barrier();
    ++i;
  }
}

// A wave's 16 columns from c0 on of rows (and columns) of scratch.
template <int N>
__device__ static inline void put_columns(const f32x4 (&x)[N], float* to, int rows, int stride, int c0, Lane l) {
  const Buffer b = buffer(to, (unsigned)(rows * stride) * 4u);
  const unsigned own = (unsigned)(4 * l.g * stride + c0 + l.i) * 4u;
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[r][j]), b, own, (unsigned)((16 * r + j) * stride) * 4u, 0);
}

template <typename T, int D1, int NW, bool VEC, bool FWD>
__device__ static __forceinline__ void scan(const Args& A) {
  constexpr int NO = Kind<T>::kOut;
  typedef Chunks<T, D1, NW, (FWD ? NO : 0)> L;
  constexpr int C = L::C, NT = C / 16, NS = C / 32, KT = D1 / 16, KS = D1 / 32, NI = L::NI, VC = 16 * NW;
  typedef typename L::MK MK;
  typedef typename L::MV MV;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int bh = blockIdx.x, col0 = blockIdx.y * VC, n = length_of(A, bh), c0 = col0 + 16 * wave, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  const Rows xk = rows_at<T>(A.K, A, bh, A.dk, n, 0, A.dk), xq = rows_at<T>(A.Q, A, bh, A.dk, n, 0, A.dk),
             xv = rows_at<T>(A.V, A, bh, A.dv, n, col0, min(A.dv - col0, VC)), xo = rows_at<T>(A.out, A, bh, A.dv, n, col0, min(A.dv - col0, VC));
  if (FWD && n < A.L) zero_rows<T>(xo, n, A.L, tid, L::kThreads);
  if (wave >= NW) {
    if (chunks > 0) load_chunks<L, T, D1, (FWD ? NO : 0), VEC, false>(A, bh, xk, xq, xv, n, tid - 64 * NW);
    return;
  }
  f32x4 S[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) S[kt] = zero4();
  if (A.s_in != nullptr) load_state<KT, true>(S, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g);
  const Bases<L> base(l, lane, wave);
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tq = base.kFar ? buf * MK::kAll : L::q + buf * MK::kAll, tv = buf * L::kV, tt = buf * L::kT, tp = buf * L::kP, tw = buf * L::kW;
    const int rb = base.rows, rq = base.query, cb = base.cols, vb = base.value, tb = base.tri, pb = base.weights, wb = base.vec, wi = base.vec_row;
    const int r0 = c * C, nr = min(C, n - r0);
    if (!FWD) put_columns<KT>(S, A.states + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), D1, A.dvp, c0, l);
    // Steps: the products of one run while the next one's operands are read and split.
    f32x4 R[NT], O[NT], U[NT], V[NT], gamma[NT], beta[NT];
#pragma unroll
    for (int r = 0; r < NT; ++r) R[r] = O[r] = U[r] = zero4();
    u32x4 t0[3][NT];
    const auto ask_row = [&](int r) {
      V[r] = MV::quad(tv, vb, 0, r);
      gamma[r] = lds_get<f32x4>(wb + tw + 4 * (16 * r));
      beta[r] = lds_get<f32x4>(wb + tw + 4 * (2 * C + 16 * r));
    };
    {
      Planes<NI> k[2][NT], q[2][NT];
      Planes<3> b[2];
      const auto ask = [&](int s) {
#pragma unroll
        for (int r = 0; r < NT; ++r) {
          k[s & 1][r] = MK::row(tk, rb, r, s);
          if (FWD) q[s & 1][r] = MK::row(tq, rq, r, s);
        }
      };
      ask(0);
      b[0] = split<3>(S[0], S[1]);
      step_end();
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if (s + 1 < KS) {
          ask(s + 1);
          b[(s + 1) & 1] = split<3>(S[2 * s + 2], S[2 * s + 3]);
        } else {
#pragma unroll
          for (int r = 0; r < 2; ++r) ask_row(r);
        }
        mma_rows<NI, 3>(k[s & 1], b[s & 1], R);
        if (FWD) mma_cols<NO, NI>(b[s & 1], q[s & 1], O);
        interleave<NI == 1 ? NT * (3 + (FWD ? NO : 0)) : 0, 3, NI == 1 ? (FWD ? 2 : 1) * NT : 0>();
      }
    }
    step_end();
    const auto correct = [&](int r) { R[r] = beta[r] * (V[r] - gamma[r] * R[r]); };
    const float Gamma = lds_get<float>(wb + tw + 4 * (3 * C));
    Planes<NI> k0[KT];
    Planes<3> bu[NS];
    f32x4 left[NT];
    {
      Planes<3> b[NS];
#pragma unroll
      for (int i = 0; i < 3; ++i) tri_plane<C, true>(tt, tb, 0, i, t0[i]);
#pragma unroll
      for (int r = 2; r < NT; ++r) ask_row(r);
      correct(0);
      correct(1);
      b[0] = split<3>(R[0], R[1]);
      step_end();
      u32x4 t1[3][NT];
      if constexpr (NS == 2) {
#pragma unroll
        for (int i = 0; i < 3; ++i) tri_plane<C, true>(tt, tb, 1, i, t1[i]);
        correct(2);
        correct(3);
        b[1] = split<3>(R[2], R[3]);
      }
      mma_step<C, true, false, 3, 3>(t0, 0, b[0], U);
      interleave<NI == 1 ? 24 : 0, 4, NI == 1 ? 6 : 0>();
#pragma unroll
      for (int r = 0; r < NT; ++r) left[r] = lds_get<f32x4>(wb + tw + 4 * (C + 16 * r));
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) k0[kt] = MK::col(tk, cb, kt, 0);
      bu[0] = split<3>(left[0] * U[0], left[1] * U[1]);
      if constexpr (NS == 2) {
        mma_step<C, true, false, 3, 3>(t1, 1, b[1], U);
        interleave<NI == 1 ? 12 : 0, 5, NI == 1 ? 2 * KT : 0>();
      } else {
        step_end();
      }
    }
    step_end();
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) S[kt] *= Gamma;
    Planes<NO> po[NS];
    Planes<NI> k1[KT];
    if constexpr (NS == 2) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) k1[kt] = MK::col(tk, cb, kt, 1);
      bu[NS - 1] = split<3>(left[2] * U[2], left[3] * U[3]);
    }
    mma_rows<NI, 3>(k0, bu[0], S);
    if constexpr (NS == 2) {
      interleave<NI == 1 ? 3 * KT : 0, 2, NI == 1 ? 2 * KT : 0>();
      mma_rows<NI, 3>(k1, bu[NS - 1], S);
    }
    if (FWD) {
      u32x4 t[NO][NT];
#pragma unroll
      for (int i = 0; i < NO; ++i) tri_plane<C, true>(tp, pb, 0, i, t[i]);
#pragma unroll
      for (int r = 0; r < NT; ++r) O[r] *= lds_get<float>(wi + tw + 4 * (16 * r));
      po[0] = split<NO>(U[0], U[1]);
      interleave<NI == 1 ? 3 * KT : 0, 2, 0>();
      mma_step<C, true, true, NO, NO>(t, 0, po[0], O);
      if constexpr (NS == 2) {
        step_end();
#pragma unroll
        for (int i = 0; i < NO; ++i) tri_plane<C, true>(tp, pb, 1, i, t[i]);
        po[1] = split<NO>(U[2], U[3]);
        mma_step<C, true, true, NO, NO>(t, 1, po[NS - 1], O);
      }
      const unsigned col = (unsigned)((16 * wave + 4 * l.g) * (int)sizeof(T));
      const Buffer ob = xo.rows(r0, nr);
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        const int row = 16 * r + l.i;
        if (VEC) buffer_quad<T>(ob, col < xo.width && row < nr ? (unsigned)row * xo.row + col : kNowhere, A.scale * O[r]);
        else if (row < nr && col < xo.width) store_quad<T>(xo.at(r0 + row) + col, (int)(xo.width - col), A.scale * O[r]);
      }
    } else {
      put_columns<NT>(U, A.u + chunk_at(A, bh, c) * ((long long)C * A.dvp), C, A.dvp, c0, l);
    }
  };
  if (chunks > 0) each_chunk<L, false>(chunks, step);
  if (A.s_out != nullptr) store_state<KT>(S, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g);
}

// ---------------------------------------------------------------------------
// From the last chunk to the first: the gradient G of the state behind each chunk, and dR.
// ---------------------------------------------------------------------------
template <typename T, int D1, int NW, bool VEC>
__device__ static __forceinline__ void scan_back(const Args& A) {
  typedef Chunks<T, D1, NW, 3> L;
  constexpr int C = L::C, NT = C / 16, NS = C / 32, KT = D1 / 16, KS = D1 / 32, NI = L::NI, VC = 16 * NW;
  typedef typename L::MK MK;
  typedef typename L::MV MV;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int bh = blockIdx.x, col0 = blockIdx.y * VC, n = length_of(A, bh), c0 = col0 + 16 * wave, chunks = (n + C - 1) / C;
  const Lane l{lane & 15, lane >> 4};
  if (wave >= NW) {
    const Rows xk = rows_at<T>(A.K, A, bh, A.dk, n, 0, A.dk), xq = rows_at<T>(A.Q, A, bh, A.dk, n, 0, A.dk),
               xo = rows_at<T>(A.dOut, A, bh, A.dv, n, col0, min(A.dv - col0, VC));
    if (chunks > 0) load_chunks<L, T, D1, 3, VEC, true>(A, bh, xk, xq, xo, n, tid - 64 * NW);
    return;
  }
  f32x4 G[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) G[kt] = zero4();
  if (A.s_in != nullptr) load_state<KT, true>(G, A.s_in + (long long)bh * A.dk * A.dv, A.dk, A.dv, 0, c0 + l.i, l.g);
  const Bases<L> base(l, lane, wave);
  const auto step = [&](int c, auto buffer_of) {
    constexpr int buf = decltype(buffer_of)::value, tk = buf * MK::kAll, tq = base.kFar ? buf * MK::kAll : L::q + buf * MK::kAll, tv = buf * L::kV, tt = buf * L::kT, tp = buf * L::kP, tw = buf * L::kW;
    const int rb = base.rows, cb = base.cols, qb = base.query_cols, vb = base.value, tb = base.tri, pb = base.weights, wb = base.vec;
    put_columns<KT>(G, A.dstates + chunk_at(A, bh, c) * ((long long)D1 * A.dvp), D1, A.dvp, c0, l);
    f32x4 U[NT], R[NT], W[NT];
#pragma unroll
    for (int r = 0; r < NT; ++r) U[r] = R[r] = W[r] = zero4();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      Planes<NI> k[NT];
#pragma unroll
      for (int r = 0; r < NT; ++r) k[r] = MK::row(tk, rb, r, s);
      mma_rows<NI, 3>(k, split<3>(G[2 * s], G[2 * s + 1]), U);
    }
    {
      Planes<NI> b[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) b[s] = MV::col(tv, vb, 0, s);
      mma_tri<C, false, false, 3, NI, 3>(tp, pb, b, W);
    }
#pragma unroll
    for (int r = 0; r < NT; ++r) U[r] = lds_get<f32x4>(wb + tw + 4 * (C + 16 * r)) * U[r] + W[r];
    {
      Planes<3> b[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) b[s] = split<3>(U[2 * s], U[2 * s + 1]);
      mma_tri<C, false, false, 3, 3, 3>(tt, tb, b, R);
    }
    {
      const float Gamma = lds_get<float>(wb + tw + 4 * (3 * C));
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) G[kt] *= Gamma;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const f32x4 w0 = lds_get<f32x4>(wb + tw + 4 * (32 * s)), w1 = lds_get<f32x4>(wb + tw + 4 * (32 * s + 16));
        const f32x4 b0 = lds_get<f32x4>(wb + tw + 4 * (2 * C + 32 * s)), b1 = lds_get<f32x4>(wb + tw + 4 * (2 * C + 32 * s + 16));
        Planes<NI> x[KT];
        {
          const Planes<3> o = split<3>(A.scale * w0 * MV::quad(tv, vb, 0, 2 * s), A.scale * w1 * MV::quad(tv, vb, 0, 2 * s + 1));
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) x[kt] = MK::col(tq, qb, kt, s);
          mma_rows<NI, 3>(x, o, G);
        }
        const Planes<3> b = split<3>(-(w0 * b0) * R[2 * s], -(w1 * b1) * R[2 * s + 1]);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) x[kt] = MK::col(tk, cb, kt, s);
        mma_rows<NI, 3>(x, b, G);
      }
    }
    {
      put_columns<NT>(R, A.dr + chunk_at(A, bh, c) * ((long long)C * A.dvp), C, A.dvp, c0, l);
    }
  };
  if (chunks > 0) each_chunk<L, true>(chunks, step);
  if (A.s_out != nullptr) store_state<KT>(G, A.s_out + (long long)bh * A.dk * A.dv, A.dk, A.dv, c0 + l.i, l.g);
}

template <typename T, int D1, int NW, bool VEC>
__global__ __launch_bounds__((Chunks<T, D1, NW, 1>::kThreads)) void k_delta_scan(Args A) {
  scan<T, D1, NW, VEC, true>(A);
}
// Backward: the gradients of the states (z = 0) and the states (z = 1) do not wait for each other.
template <typename T, int D1, int NW, bool VEC>
__global__ __launch_bounds__((Chunks<T, D1, NW, 3>::kThreads)) void k_delta_back(Args A, const float* g_in, float* g_out) {
  if (blockIdx.z == 0) {
    A.s_in = g_in;
    A.s_out = g_out;
    scan_back<T, D1, NW, VEC>(A);
  } else {
    scan<T, D1, NW, VEC, false>(A);
  }
}

// ---------------------------------------------------------------------------
// Launches: the instance that holds dk inner values.
// ---------------------------------------------------------------------------
template <typename T>
static bool vec_of(const Args& a) { return a.dk * sizeof(T) % 16 == 0 && a.dv * sizeof(T) % 16 == 0; }

template <typename T, int D1, bool VEC, bool BWD>
static dark_status go_prep(const Args& a, hipStream_t st) {
  constexpr int lds = prep_lds<T, D1>();
  DARK_TRY(allow_lds(k_delta_prep<T, D1, VEC, BWD>, lds));
  DARK_LAUNCH(KID_DELTA_PREP, st, (k_delta_prep<T, D1, VEC, BWD>), dim3((unsigned)(a.B * a.H * a.chunks)), dim3(256), lds, a);
  return DARK_OK;
}
template <typename T, int D1>
static dark_status go_prep(const Args& a, bool backward, hipStream_t st) {
  if (vec_of<T>(a)) return backward ? go_prep<T, D1, true, true>(a, st) : go_prep<T, D1, true, false>(a, st);
  return backward ? go_prep<T, D1, false, true>(a, st) : go_prep<T, D1, false, false>(a, st);
}
template <typename T>
static dark_status launch_prep(const Args& a, bool backward, hipStream_t st) {
  switch (inner_of(a.dk)) {
    case 64: return go_prep<T, 64>(a, backward, st);
    case 128: return go_prep<T, 128>(a, backward, st);
    default: return go_prep<T, 256>(a, backward, st);
  }
}

// 256 rows of a state leave room for one wave a SIMD.
template <int D1>
constexpr int waves_of() { return D1 > 128 ? 2 : 4; }

template <typename T, int D1, int NW, bool VEC>
static dark_status go_scan(const Args& a, hipStream_t st) {
  typedef Chunks<T, D1, NW, Kind<T>::kOut> L;
  DARK_TRY(allow_lds(k_delta_scan<T, D1, NW, VEC>, L::all));
  DARK_LAUNCH(KID_DELTA_SCAN, st, (k_delta_scan<T, D1, NW, VEC>), dim3(a.B * a.H, (a.dv + 16 * NW - 1) / (16 * NW)), dim3(L::kThreads), L::all, a);
  return DARK_OK;
}
template <typename T, int D1, int NW, bool VEC>
static dark_status go_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  typedef Chunks<T, D1, NW, 3> L;
  constexpr int lds = L::all > Chunks<T, D1, NW, 0>::all ? L::all : Chunks<T, D1, NW, 0>::all;
  DARK_TRY(allow_lds(k_delta_back<T, D1, NW, VEC>, lds));
  DARK_LAUNCH(KID_DELTA_BACK, st, (k_delta_back<T, D1, NW, VEC>), dim3(a.B * a.H, a.dvp / (16 * NW), states ? 2 : 1), dim3(L::kThreads), lds, a, g_in, g_out);
  return DARK_OK;
}
template <typename T, int D1>
static dark_status go_scan(const Args& a, hipStream_t st) {
  constexpr int NW = waves_of<D1>();
  return vec_of<T>(a) ? go_scan<T, D1, NW, true>(a, st) : go_scan<T, D1, NW, false>(a, st);
}
template <typename T, int D1>
static dark_status go_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  constexpr int NW = waves_of<D1>();
  return vec_of<T>(a) ? go_back<T, D1, NW, true>(a, g_in, g_out, states, st) : go_back<T, D1, NW, false>(a, g_in, g_out, states, st);
}
template <typename T>
static dark_status launch_scan(const Args& a, hipStream_t st) {
  switch (inner_of(a.dk)) {
    case 64: return go_scan<T, 64>(a, st);
    case 128: return go_scan<T, 128>(a, st);
    default: return go_scan<T, 256>(a, st);
  }
}
template <typename T>
static dark_status launch_back(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  switch (inner_of(a.dk)) {
    case 64: return go_back<T, 64>(a, g_in, g_out, states, st);
    case 128: return go_back<T, 128>(a, g_in, g_out, states, st);
    default: return go_back<T, 256>(a, g_in, g_out, states, st);
  }
}

}  // namespace delta
}  // namespace dark
