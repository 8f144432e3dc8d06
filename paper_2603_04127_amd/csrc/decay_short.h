// The scan of decayed linear attention (decay.h) for short sequences, in one launch and without a state: every block of 64 rows sums
// over the keys before it, P = x1 x2^T decayed, y = P x3, in chunks of 64 keys.  The work grows with the square of the length, but no
// chunk waits for another one's state, and one launch does what takes three on long sequences.  The state behind the sequence, where
// it is asked for, is summed up by workgroups of their own in the same launch.
//
// Eight waves are two groups of four; a group takes every second chunk of keys, and the groups' sums are joined at the end: half
// as many steps one after the other.  In a group each wave holds 16 rows of x1 as operands in registers.  P^T comes out of the matrix
// unit with the keys along a lane's registers and goes back in as an operand after two exchanges between lane groups.
// Bound by the chain of a block's chunks, two of them in 1.4 to 2.9 us: 16 heads of 777 x 128 take 20 us (24 as segments), 24 of 512 x 64 11
// (17).  More groups shorten the chain and take their turns on the same SIMDs: four are no faster there (four of half the rows 20 us, four
// of all 20.4) and slower elsewhere.
#pragma once

#include "decay_scan.h"

namespace dark {
namespace decay {

// x1 rows as operands straight from memory: eight values of the lane's row for every 32.
template <typename T, int D1, bool VEC>
__device__ static inline void load_rows(typename Op<T>::frag (&x)[D1 / 32], const Rows& rows, int r0, int nr, int r, int g) {
  static_assert(sizeof(T) == 2, "bf16");
  const unsigned at = rows.offset(r, nr);
  if (VEC) {
    const Buffer b = rows.rows(r0, nr);
#pragma unroll
    for (int k = 0; k < D1 / 32; ++k) {
      const unsigned c = (unsigned)(32 * k + 8 * g) * 2u;
      x[k] = __builtin_amdgcn_raw_buffer_load_b128(b, c < rows.width ? at + c : kNowhere, 0, 0);
    }
  } else {
    unsigned skew;
    const Buffer b = rows.loose(r0, nr, skew);
    Piece<T> p[D1 / 32];
#pragma unroll
    for (int k = 0; k < D1 / 32; ++k) {
      const unsigned c = (unsigned)(32 * k + 8 * g) * 2u;
      p[k].load(b, c < rows.width && r < nr ? at + c + skew : kNowhere);
    }
#pragma unroll
    for (int k = 0; k < D1 / 32; ++k) x[k] = p[k].get(((at + skew) >> 1 & 1u) * 16u, (int)rows.width - (32 * k + 8 * g) * 2);
  }
}

template <typename T, int D1, int D2>
constexpr int short_lds() { return 64 * 2 * (D1 + D2) * (int)sizeof(T) + 3 * 64 * 4; }

template <typename T, int D1, int D2, bool VEC>
__global__ __launch_bounds__(512, 2) void k_decay_short(Scans A, int blocks, int state_blocks) {
  typedef Op<T> O;
  constexpr int C = 64, RB1 = D1 * (int)sizeof(T), RB2 = D2 * (int)sizeof(T), K1 = D1 / 32, CT = D2 / 16, KT = D1 / 16;
  constexpr int tile = C * (RB1 + RB2), tw = 2 * tile, tl = tw + 4 * C, tk = tl + 4 * C;
  const int tid = threadIdx.x, gtid = tid & 255, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, group = __builtin_amdgcn_readfirstlane(tid >> 8);
  const int t2 = group * tile, t3 = t2 + C * RB1;
  Scan a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  if (blockIdx.z == 2) a = A.s[2];
  const int heads = A.B * A.H, states = heads * state_blocks;
  const bool summing = (int)blockIdx.x < states;   // the state's workgroups come first: they take the longest
  const int at = summing ? (int)blockIdx.x : (int)blockIdx.x - states;
  const int bh = summing ? at / state_blocks : at % heads, b = bh / A.H, h = bh % A.H;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const float a2 = decay_log2(A.log_decay, h);
  const Rows x2 = rows_of<T>(a.x2, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n, 0, a.d1);
  const Lane l = {lane & 15, lane >> 4};
  const long long uat = (long long)bh * a.d1 * a.d2;

  if (summing) {
    const int col0 = blockIdx.y * D2 + 64 * (at % state_blocks), cols = min(a.d2 - col0, 64);
    if (a.u_out == nullptr || cols <= 0) return;
    const Rows x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
    const int chunks = (n + C - 1) / C, steps = (chunks + 1) / 2;
    put_weights<C>(tw, a2, C, a.off, a.su, tid);
    put_weights<C>(tl, a2, n - (chunks - 1) * C, a.off, a.su, tid);   // the last chunk's
    Tile<T, C, D1, 256, VEC> p2;
    Tile<T, C, 64, 256, VEC> p3;
    const auto load = [&](int c) {
      const int nr = min(C, n - c * C);   // none behind the last chunk
      p2.load(x2, c * C, max(nr, 0), gtid);
      p3.load(x3, c * C, max(nr, 0), gtid);
    };
    load(group);
    f32x4 U[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) U[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < steps; ++s) {
      const int c = 2 * s + group;
      lds_barrier();
      p2.store(t2, gtid);
      p3.store(t3, gtid);
      lds_barrier();
      load(c + 2);
      if (c < chunks) update<T, C, D1, 64>(U, t2, t3, c == chunks - 1 ? tl : tw, power(a2, max(n - (c + 1) * C, 0)), wave, fresh<VEC && D2 <= 64 ? D1 : 128>(lane));
    }
    lds_barrier();
    const int mine = (wave * KT * 64 + lane) * 16;
    if (group == 1) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) lds_put(mine + kt * 1024, U[kt]);
    }
    lds_barrier();
    if (group == 1) return;
    f32x4 first[KT];
    const int uc = col0 + 16 * wave + l.i;
    if (a.u_in != nullptr) {
      load_state<KT, VEC>(first, a.u_in + uat, a.d1, a.d2, a.transposed, uc, l.g);
    } else {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) first[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float gn = power(a2, n);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) U[kt] = U[kt] + lds_get<f32x4>(mine + kt * 1024) + gn * first[kt];
    store_state<KT>(U, a.u_out + uat, a.d1, a.d2, uc, l.g);
    return;
  }

  if (a.y == nullptr) return;
  const int qb = blocks - 1 - at / heads, begin = qb * C, end = min(begin + C, A.L), col0 = blockIdx.y * D2, cols = min(a.d2 - col0, D2);
  if (cols <= 0) return;   // a narrower scan than another one of the launch
  if (end > n) {   // rows behind the sequence
    const Rows y = rows_of<T>(a.y, b, h, A.H, A.L, a.d2, A.layout, 0, n, col0, cols);
    for (int r = max(begin, n) + (tid >> 6); r < end; r += 8)
      for (int c = lane; c < cols; c += 64) reinterpret_cast<T*>(const_cast<char*>(y.head) + (long long)r * y.row)[c] = (T)0;
    if (begin >= n) return;
  }
  const int nr = min(C, n - begin);
  const Rows x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
  Tile<T, C, D1, 256, VEC> p2;
  Tile<T, C, D2, 256, VEC> p3;
  const auto load = [&](int kb) {   // no rows where there is no such chunk
    const int k = max(kb, 0), rows = kb >= 0 ? min(C, n - kb * C) : 0;
    p2.load(x2, k * C, rows, gtid);
    p3.load(x3, k * C, rows, gtid);
  };
  load(qb - group);
  typename O::frag x1[K1];
  load_rows<T, D1, VEC>(x1, rows_of<T>(a.x1, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n, 0, a.d1), begin, nr, 16 * wave + l.i, l.g);
  if (tid < C) lds_put(tk + 4 * tid, power(a2, C - 1 - tid));
  f32x4 out[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) out[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int q = 16 * wave + l.i;   // the lane's row in the block
  if (a.u_in != nullptr) {
    // the state as a tile of D1 rows, rounded to bf16 (its product goes into an output of that type); each group takes half of the rows
    const Buffer u = buffer(a.u_in + uat, (unsigned)(a.d1 * a.d2) * 4u);
    constexpr int kAtOnce = 8;
    for (int e0 = 0; e0 < D1 * D2; e0 += 512 * kAtOnce) {
      float v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int e = e0 + 512 * i + tid, r = a.transposed ? e % D1 : e / D2, c = col0 + (a.transposed ? e / D1 : e % D2);
        v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(u, r < a.d1 && c < a.d2 ? (unsigned)(a.transposed ? c * a.d1 + r : r * a.d2 + c) * 4u : kNowhere, 0, 0));
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int e = e0 + 512 * i + tid, r = a.transposed ? e % D1 : e / D2, c = a.transposed ? e / D1 : e % D2;
        lds_put(r * RB2 + (((c / 8) ^ swz<RB2>(r)) << 4) + 2 * (c & 7), (unsigned short)pack_bf16(v[i], 0.f));
      }
    }
    lds_barrier();
    const int bc = O::template col_base<RB2>(l);
#pragma unroll
    for (int k = 0; k < K1 / 2; ++k) {
      const int rows = 32 * (group * (K1 / 2) + k) * RB2;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) out[ct] = O::mma(O::template col<RB2>(rows, bc, ct), group == 0 ? x1[k] : x1[K1 / 2 + k], out[ct]);
    }
    const float lead = a.sr * power(a2, begin + q + 1 - a.off);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) out[ct] *= lead;
  }

  const int steps = qb / 2 + 1;
  for (int s = 0; s < steps; ++s) {
    const int kb = qb - group - 2 * s;   // from the nearest chunk on
    lds_barrier();
    p2.store(t2, gtid);
    p3.store(t3, gtid);
    lds_barrier();
    load(s + 1 < steps ? kb - 2 : -1);
    if (kb < 0) continue;
    const Lane f = fresh<VEC && D2 <= 64 ? D1 : 128>(lane);
    const int br = O::template row_base<RB1>(f);
    typename O::frag p[2];
    // g^(r-c) with r - c = 64 (qb - kb) - 63 + q + (63 - key): both factors have exponents >= 0 except on the diagonal
    const float near = kb < qb ? a.sp * power(a2, C * (qb - kb) - (C - 1) + q) : a.sp;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      f32x4 st[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int kt = 2 * ks + i;
#pragma unroll
        for (int k = 0; k < K1; ++k) st[i] = O::mma(O::row(t2 + kt * 16 * RB1, br, k), x1[k], k > 0 ? st[i] : f32x4{0.f, 0.f, 0.f, 0.f});
        if (kb < qb) {
          st[i] *= near * lds_get<f32x4>(tk + 64 * kt + 16 * f.g);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int apart = q - 16 * kt - 4 * f.g - j;
            st[i][j] = apart >= 0 ? st[i][j] * (near * power(a2, max(apart, 0))) : 0.f;
          }
        }
      }
      p[ks] = O::state(st[0], st[1]);
      hold();
    }
    const int bc = O::template col_base<RB2>(f);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) out[ct] = O::mma(O::template col<RB2>(t3 + 32 * ks * RB2, bc, ct), p[ks], out[ct]);
      if (ct % 4 == 3) hold();
    }
  }
  lds_barrier();
  const int mine = (wave * CT * 64 + lane) * 16;
  if (group == 1) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) lds_put(mine + ct * 1024, out[ct]);
  }
  lds_barrier();
  if (group == 1) return;
  const Rows y = rows_of<T>(a.y, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
  const Buffer yb = y.rows(begin, nr);
  const unsigned row = y.offset(q, nr);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const f32x4 v = out[ct] + lds_get<f32x4>(mine + ct * 1024);
    const unsigned c = (unsigned)((16 * ct + 4 * l.g) * (int)sizeof(T));
    if (VEC) {
      O::store4(yb, c < y.width ? row + c : kNowhere, v);
    } else if (q < nr && c < y.width) {
      O::store_loose(y.at(begin + q) + c, (int)(y.width - c), v);
    }
  }
}

template <typename T, int D1, int D2, bool VEC>
static dark_status launch_short(const Scans& a, int n, hipStream_t st) {
  constexpr int lds = short_lds<T, D1, D2>();
  DARK_TRY(allow_lds(k_decay_short<T, D1, D2, VEC>, lds));
  bool out = false, rows = false;
  for (int i = 0; i < n; ++i) {
    out = out || a.s[i].u_out != nullptr;
    rows = rows || a.s[i].y != nullptr;
  }
  int d1, d2;
  widths_of(a, n, &d1, &d2);
  const int blocks = rows ? (a.L + 63) / 64 : 0, states = out ? ((d2 < D2 ? d2 : D2) + 63) / 64 : 0;
  const dim3 grid((unsigned)(a.B * a.H * (blocks + states)), (unsigned)((d2 + D2 - 1) / D2), (unsigned)n);
  if (grid.x == 0) return DARK_OK;
  DARK_LAUNCH(KID_DECAY_SHORT, st, (k_decay_short<T, D1, D2, VEC>), grid, dim3(512), lds, a, blocks, states);
  return DARK_OK;
}
template <typename T, int D1, int D2>
static dark_status pick_short(const Scans& a, int n, hipStream_t st) {
  const bool vec = a.s[0].d1 * sizeof(T) % 16 == 0 && a.s[0].d2 * sizeof(T) % 16 == 0;
  return vec ? launch_short<T, D1, D2, true>(a, n, st) : launch_short<T, D1, D2, false>(a, n, st);
}
template <typename T>
static dark_status pick_short(const Scans& a, int n, hipStream_t st) {
  int d1, d2;
  widths_of(a, n, &d1, &d2);
  if (d1 > 128) return pick_short<T, 256, 64>(a, n, st);
  if (d1 > 64) return d2 <= 64 ? pick_short<T, 128, 64>(a, n, st) : pick_short<T, 128, 128>(a, n, st);
  return d2 <= 64 ? pick_short<T, 64, 64>(a, n, st) : pick_short<T, 64, 128>(a, n, st);
}

}  // namespace decay
}  // namespace dark
