// The gated delta rule's gradients of a chunk from its state, the gradient of the state behind it, U and dR (see delta.h).
#pragma once

#include "delta_tile.h"

namespace dark {
namespace delta {

// Columns of states, U, dR, dO and V that are taken at a time.
constexpr int kBlock = 64;

template <typename T, int D1>
struct GradLds {
  static constexpr int C = Kind<T>::kChunk, NI = Kind<T>::kIn, NP = Kind<T>::kOut;
  static constexpr int NW = D1 == 64 ? 4 : 8;   // waves
  typedef Mat<C, D1, NI> MK;
  typedef Mat<C, kBlock, NI> MO;
  typedef Mat<C, kBlock, 3> MU;
  typedef Mat<C, 64, NP> MX;   // N and M, a row for every key; of 64 columns (C of them used)
  static constexpr int k = 0, q = k + MK::kAll, o = q + MK::kAll, u = o + MO::kAll, d = u + MU::kAll, behind = d + MU::kAll;
  static constexpr int n = o, m = n + MX::kAll;   // in the place of dO, U and dR
  static constexpr int w = behind > m + MX::kAll ? behind : m + MX::kAll;
  static constexpr int cross = w + kVecs * C * 4;           // [C / 16][C]
  static constexpr int third = cross + (C / 16) * C * 4;    // [C]
  static constexpr int vdot = third + C * 4;                // [C]
  static constexpr int dots = vdot + C * 4;                 // [NW][3][C]
  static constexpr int total = dots + 3 * NW * C * 4;       // [NW]
  static constexpr int all = total + 4 * NW;
};

// Sums over the lanes of a row of 16 up to each of them.
__device__ static inline float row16_prefix(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, true));
  return v;
}

// A chunk by four or eight waves, two a SIMD: each computes its share of the dk columns of dQ and dK, transposed, so that a lane has four neighbouring columns of
// a row.  The products with the states go over their dv columns in blocks; the states' operands come straight from memory, since
// no two waves need the same rows of them.
// 1536 chunks of 64 x 64 in bf16 take 64 us: 120 KB each, two thirds of it states, their gradients, U and dR in fp32, 3.1 TB/s, with the waves waiting half of their
// cycles; 576 of 64 x 128 48 to 57.  Four
// waves where there are columns for eight (dk of 128) took 69, and operands of all steps at once 78 instead of 65 (dk of 64).
template <typename T, int D1, bool VEC>
__global__ __launch_bounds__((64 * GradLds<T, D1>::NW), 2) void k_delta_grad(Args A) {
  typedef GradLds<T, D1> L;
  constexpr int C = L::C, NT = C / 16, NI = L::NI, NW = L::NW, NTH = 64 * NW, DT = D1 / 16 / NW, NP = L::NP;
  typedef typename L::MK MK;
  typedef typename L::MO MO;
  typedef typename L::MU MU;
  typedef typename L::MX MX;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int bh = blockIdx.x / A.chunks, c = blockIdx.x % A.chunks, r0 = c * C, n = length_of(A, bh), nr = min(C, n - r0), rows = min(C, A.L - r0);
  const Lane l{lane & 15, lane >> 4};
  const Rows xk = rows_at<T>(A.K, A, bh, A.dk, n, 0, A.dk), xq = rows_at<T>(A.Q, A, bh, A.dk, n, 0, A.dk);
  const Rows yq = rows_at<T>(A.dQ, A, bh, A.dk, n, 0, A.dk), yk = rows_at<T>(A.dK, A, bh, A.dk, n, 0, A.dk), yv = rows_at<T>(A.dV, A, bh, A.dv, n, 0, A.dv);
  // rows behind the sequence
  if (nr < rows) {
    const int begin = max(n, r0);
    if (A.dQ != nullptr) zero_rows<T>(yq, begin, r0 + rows, tid, NTH);
    if (A.dK != nullptr) zero_rows<T>(yk, begin, r0 + rows, tid, NTH);
    if (A.dV != nullptr) zero_rows<T>(yv, begin, r0 + rows, tid, NTH);
    for (int t = begin + tid; t < r0 + rows; t += NTH) {
      if (A.dgate != nullptr) A.dgate[gate_at(A, bh, t)] = 0.f;
      if (A.dbeta != nullptr) A.dbeta[gate_at(A, bh, t)] = 0.f;
    }
  }
  if (nr <= 0) return;
  {
    Load<T, C, D1, NTH, VEC> lk, lq;
    lk.load(xk, r0, nr, tid);
    lq.load(xq, r0, nr, tid);
    for (int e = tid; e < kVecs * C; e += NTH) lds_put(L::w + 4 * e, A.vec[chunk_at(A, bh, c) * (kVecs * C) + e]);
    lk.template store<MK>(L::k, tid);
    lq.template store<MK>(L::q, tid);
  }
  const float* const states = A.states + chunk_at(A, bh, c) * ((long long)D1 * A.dvp);
  const float* const dstates = A.dstates + chunk_at(A, bh, c) * ((long long)D1 * A.dvp);
  const float* const us = A.u + chunk_at(A, bh, c) * ((long long)C * A.dvp);
  const float* const drs = A.dr + chunk_at(A, bh, c) * ((long long)C * A.dvp);

  f32x4 X1[DT][NT], X2[DT][NT], X3[DT][NT];   // (dO S^T)^T, (dR S^T)^T, (U dS'^T)^T
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < NT; ++r) X1[i][r] = X2[i][r] = X3[i][r] = zero4();
  f32x4 N[NT], F[NT];   // of row tile `wave`: dO U^T, dR U^T
#pragma unroll
  for (int r = 0; r < NT; ++r) N[r] = F[r] = zero4();
  float sg = 0.f;                                   // <S, dS'>
  constexpr int kUnits = C * kBlock / 8, kEach = (kUnits + NTH - 1) / NTH;   // C = 32: units for half of eight waves
  float vdot[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) vdot[e] = 0.f;
  const int ob = MO::row_base(l);
#pragma unroll 1
  for (int b0 = 0; b0 < A.dvp; b0 += kBlock) {
    const Rows xo = rows_at<T>(A.dOut, A, bh, A.dv, n, b0, min(A.dv - b0, kBlock)), xv = rows_at<T>(A.V, A, bh, A.dv, n, b0, min(A.dv - b0, kBlock));
    Load<T, C, kBlock, NTH, VEC> lo, lv;
    lo.load(xo, r0, nr, tid);
    lv.load(xv, r0, nr, tid);
    f32x4 u[kEach][2], d[kEach][2];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int x = tid + e * NTH, at = (x / 8) * A.dvp + b0 + (x % 8) * 8;
      if (kUnits % NTH != 0 && x >= kUnits) break;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u[e][k] = *reinterpret_cast<const f32x4*>(us + at + 4 * k);
        d[e][k] = *reinterpret_cast<const f32x4*>(drs + at + 4 * k);
      }
    }
    __syncthreads();
    lo.template store<MO>(L::o, tid);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int x = tid + e * NTH, row = x / 8;
      if (kUnits % NTH != 0 && x >= kUnits) break;
      MU::put8(L::u, row, x % 8, split<3>(u[e][0], u[e][1]));
      MU::put8(L::d, row, x % 8, split<3>(d[e][0], d[e][1]));
      // dR . v, and dV = beta dR
      const Planes<NI> v = lv.get(e);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo2 = 0.f, hi2 = 0.f;
#pragma unroll
        for (int p = NI - 1; p >= 0; --p) {
          lo2 += __uint_as_float(v.p[p][i] << 16);
          hi2 += __uint_as_float(v.p[p][i] & 0xffff0000u);
        }
        dot += lo2 * d[e][i >> 1][2 * (i & 1)] + hi2 * d[e][i >> 1][2 * (i & 1) + 1];
      }
      vdot[e] += dot;
      if (A.dV != nullptr && row < nr) {
        const float beta = lds_get<float>(L::w + 4 * (2 * C + row));
        const int left = ((int)A.dv - b0 - (x % 8) * 8) * (int)sizeof(T);
        char* const p = yv.at(r0 + row) + (long long)(b0 + (x % 8) * 8) * (int)sizeof(T);
        if (left > 0) store_quad<T>(p, left, beta * d[e][0]);
        if (left > 4 * (int)sizeof(T)) store_quad<T>(p + 4 * sizeof(T), left - 4 * (int)sizeof(T), beta * d[e][1]);
      }
    }
    __syncthreads();
#pragma unroll 1
    for (int s = 0; s < kBlock / 32; ++s) {   // one after the other: the registers of two steps are not there
      Planes<3> S[DT], G[DT];
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const long long at = (long long)(16 * (wave * DT + i) + l.i) * A.dvp + b0 + 32 * s + 4 * l.g;
        const f32x4 s0 = *reinterpret_cast<const f32x4*>(states + at), s1 = *reinterpret_cast<const f32x4*>(states + at + 16);
        const f32x4 g0 = *reinterpret_cast<const f32x4*>(dstates + at), g1 = *reinterpret_cast<const f32x4*>(dstates + at + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) sg += s0[j] * g0[j] + s1[j] * g1[j];
        S[i] = split<3>(s0, s1);
        G[i] = split<3>(g0, g1);
      }
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        const Planes<NI> o = MO::row(L::o, ob, r, s);
        const Planes<3> dr = MU::row(L::d, ob, r, s), uu = MU::row(L::u, ob, r, s);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          X1[i][r] = mma(S[i], o, X1[i][r]);
          X2[i][r] = mma(S[i], dr, X2[i][r]);
          X3[i][r] = mma(G[i], uu, X3[i][r]);
        }
      }
      if (wave < NT) {
        const Planes<NI> o = MO::row(L::o, ob, wave, s);
        const Planes<3> dr = MU::row(L::d, ob, wave, s);
#pragma unroll
        for (int r = 0; r < NT; ++r)
          if (r <= wave) {
            const Planes<3> uu = MU::row(L::u, ob, r, s);
            N[r] = mma(o, uu, N[r]);
            F[r] = mma(dr, uu, F[r]);
          }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    float v = vdot[e];
    v += __shfl_xor(v, 1, 64);
    v += __shfl_xor(v, 2, 64);
    v += __shfl_xor(v, 4, 64);
    if ((tid & 7) == 0 && (kUnits % NTH == 0 || tid + e * NTH < kUnits)) lds_put(L::vdot + 4 * ((tid + e * NTH) / 8), v);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sg += __shfl_xor(sg, o, 64);
  if (lane == 0) lds_put(L::total + 4 * wave, sg);
  __syncthreads();   // dO, U and dR are done with

  const int rb = MK::row_base(l), cb = MK::col_base(l), xb = MX::row_base(l), xc = MX::col_base(l);
  if (wave < NT) {
    const f32x4 be = lds_get<f32x4>(L::w + 4 * (2 * C + 16 * wave + 4 * l.g)), hs = lds_get<f32x4>(L::w + 4 * (4 * C + 16 * wave + 4 * l.g)),
                ls = lds_get<f32x4>(L::w + 4 * (5 * C + 16 * wave + 4 * l.g));
    f32x4 before = zero4(), third = zero4();   // before: Z over the key tiles that are done
    // Z_ri: the weight exp(G_r - G_i) times its gradient.  The gate of row t has those with i < t <= r: sums over the keys up to each, and over
    // the rows behind it (never differences of longer sums, whose rounding a small gradient would not survive).
#pragma unroll
    for (int r = 0; r < NT; ++r) {   // key tile
      if (r > wave) {
        if (r == wave + 1 && (wave & 1) == 0) {   // right of the diagonal, taken in by operands of 32
          MX::put_row_quad(L::n, xb, r, wave, zero4());
          MX::put_row_quad(L::m, xb, r, wave, zero4());
        }
        lds_put(L::cross + 4 * (wave * C + 16 * r + l.i), 0.f);
        continue;
      }
      f32x4 kk = zero4(), qk = zero4();
#pragma unroll
      for (int s = 0; s < D1 / 32; ++s) {
        const Planes<NI> b = MK::row(L::k, rb, r, s);
        kk = mma(MK::row(L::k, rb, wave, s), b, kk);
        qk = mma(MK::row(L::q, rb, wave, s), b, qk);
      }
      const int i = 16 * r + l.i;
      const float hi = lds_get<float>(L::w + 4 * (4 * C + i)), lo = lds_get<float>(L::w + 4 * (5 * C + i));
      f32x4 nn, mm;
      float cz = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = 16 * wave + 4 * l.g + j;
        const float d = t >= i ? expf((hs[j] - hi) + (ls[j] - lo)) : 0.f;
        const bool below = t > i;
        const float x = t >= i ? A.scale * d * N[r][j] : 0.f, f = below ? d * F[r][j] : 0.f;
        nn[j] = x;
        mm[j] = -be[j] * f;
        const float kf = kk[j] * f, z = below ? qk[j] * x - be[j] * kf : 0.f;
        third[j] += kf;
        const float up = before[j] + row16_prefix(z);
        before[j] += row16_sum(z);
        cz += below ? up : 0.f;
      }
      MX::put_row_quad(L::n, xb, r, wave, nn);
      MX::put_row_quad(L::m, xb, r, wave, mm);
      cz += xor16(cz);
      cz += xor32(cz);
      if (l.g == 0) lds_put(L::cross + 4 * (wave * C + i), cz);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float t3 = row16_sum(third[j]);
      if (l.i == 0) lds_put(L::third + 4 * (16 * wave + 4 * l.g + j), t3);
    }
  }
  // the states' part of dQ and dK, and what the gates take of it
#pragma unroll
  for (int r = 0; r < NT; ++r) {
    const float gamma = lds_get<float>(L::w + 4 * (16 * r + l.i)), leftw = lds_get<float>(L::w + 4 * (C + 16 * r + l.i)),
                beta = lds_get<float>(L::w + 4 * (2 * C + 16 * r + l.i));
    float dq = 0.f, d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const f32x4 q = MK::row_quad(L::q, rb, r, wave * DT + i), k = MK::row_quad(L::k, rb, r, wave * DT + i);
      X1[i][r] *= A.scale * gamma;
      X2[i][r] *= gamma;
      X3[i][r] *= leftw;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dq += q[j] * X1[i][r][j];
        d1 += k[j] * X2[i][r][j];
        d2 += k[j] * X3[i][r][j];
      }
      X3[i][r] -= beta * X2[i][r];
    }
    dq += xor16(dq);
    d1 += xor16(d1);
    d2 += xor16(d2);
    dq += xor32(dq);
    d1 += xor32(d1);
    d2 += xor32(d2);
    if (l.g == 0) {
      lds_put(L::dots + 4 * ((wave * 3 + 0) * C + 16 * r + l.i), dq);
      lds_put(L::dots + 4 * ((wave * 3 + 1) * C + 16 * r + l.i), d1);
      lds_put(L::dots + 4 * ((wave * 3 + 2) * C + 16 * r + l.i), d2);
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int s = 0; s < C / 32; ++s) {
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const Planes<NI> k = MK::col(L::k, cb, wave * DT + i, s), q = MK::col(L::q, cb, wave * DT + i, s);
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        if (C == 32 || r >= 2 * s) {   // rows r, keys of step s
          X1[i][r] = mma_of<NI, NP>(k, MX::col(L::n, xc, r, s), X1[i][r]);
          X3[i][r] = mma_of<NI, NP>(k, MX::col(L::m, xc, r, s), X3[i][r]);
        }
        if (C == 32 || r <= 2 * s + 1) {   // keys r, rows of step s
          X3[i][r] = mma_of<NI, NP>(k, MX::row(L::m, xb, r, s), X3[i][r]);
          X3[i][r] = mma_of<NI, NP>(q, MX::row(L::n, xb, r, s), X3[i][r]);
        }
      }
    }
  }
  const Buffer bq = yq.rows(r0, A.dQ != nullptr ? nr : 0), bk = yk.rows(r0, A.dK != nullptr ? nr : 0);
#pragma unroll
  for (int i = 0; i < DT; ++i) {
    const unsigned col = (unsigned)((16 * (wave * DT + i) + 4 * l.g) * (int)sizeof(T));
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      const int row = 16 * r + l.i;
      if (VEC) {
        const unsigned at = col < yq.width && row < nr ? (unsigned)row * yq.row + col : kNowhere;
        buffer_quad<T>(bq, at, X1[i][r]);
        buffer_quad<T>(bk, at, X3[i][r]);
      } else if (col < yq.width && row < nr) {
        if (A.dQ != nullptr) store_quad<T>(yq.at(r0 + row) + col, (int)(yq.width - col), X1[i][r]);
        if (A.dK != nullptr) store_quad<T>(yk.at(r0 + row) + col, (int)(yk.width - col), X3[i][r]);
      }
    }
  }
  if (wave == 0 && (A.dgate != nullptr || A.dbeta != nullptr)) {
    const int t = lane < C ? lane : 0;
    double dq = 0.0, d1 = 0.0, d2 = 0.0, cross = 0.0;
    for (int w = 0; w < NW; ++w) {
      dq += lds_get<float>(L::dots + 4 * ((w * 3 + 0) * C + t));
      d1 += lds_get<float>(L::dots + 4 * ((w * 3 + 1) * C + t));
      d2 += lds_get<float>(L::dots + 4 * ((w * 3 + 2) * C + t));
      if (w < NT && t > 0) cross += lds_get<float>(L::cross + 4 * (w * C + t - 1));
    }
    // reads of the state by the rows from t on, what the keys before t leave in the next one, and the state that passes through
    double reads = lane < C ? dq - (double)lds_get<float>(L::w + 4 * (2 * C + t)) * d1 : 0.0, left = lane < C ? d2 : 0.0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_down(reads, o, 64), y = __shfl_up(left, o, 64);
      if (lane + o < 64) reads += x;
      if (lane >= o) left += y;
    }
    left = __shfl_up(left, 1, 64);
    if (lane == 0) left = 0.0;
    double total = 0.0;
    for (int w = 0; w < NW; ++w) total += lds_get<float>(L::total + 4 * w);
    const double gate = reads + left + cross + total * (double)lds_get<float>(L::w + 4 * (3 * C));
    if (lane < nr) {
      if (A.dgate != nullptr) A.dgate[gate_at(A, bh, r0 + lane)] = (float)gate;
      if (A.dbeta != nullptr) A.dbeta[gate_at(A, bh, r0 + lane)] = lds_get<float>(L::vdot + 4 * t) - (float)d1 - lds_get<float>(L::third + 4 * t);
    }
  }
}

template <typename T, int D1, bool VEC>
static dark_status go_grad(const Args& a, hipStream_t st) {
  constexpr int lds = GradLds<T, D1>::all;
  DARK_TRY(allow_lds(k_delta_grad<T, D1, VEC>, lds));
  DARK_LAUNCH(KID_DELTA_GRAD, st, (k_delta_grad<T, D1, VEC>), dim3((unsigned)(a.B * a.H * a.chunks)), dim3(64 * GradLds<T, D1>::NW), lds, a);
  return DARK_OK;
}
template <typename T>
static dark_status launch_grad(const Args& a, hipStream_t st) {
  const bool vec = a.dk * sizeof(T) % 16 == 0 && a.dv * sizeof(T) % 16 == 0;
  switch (inner_of(a.dk)) {
    case 64: return vec ? go_grad<T, 64, true>(a, st) : go_grad<T, 64, false>(a, st);
    case 128: return vec ? go_grad<T, 128, true>(a, st) : go_grad<T, 128, false>(a, st);
    default: return vec ? go_grad<T, 256, true>(a, st) : go_grad<T, 256, false>(a, st);
  }
}

}  // namespace delta
}  // namespace dark
