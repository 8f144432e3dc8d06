// Operands of the gated delta rule's products: sums of bf16 planes, tiles of them in LDS.
#pragma once

#include "delta.h"

namespace dark {
namespace delta {

using namespace fz;
using namespace rows;

// A product's operand over 32 inner values, as a sum of N bf16 operands.  The products run on the matrix units in bf16 with fp32 sums; a
// 32-bit value is three truncated planes of eight bits (what is left behind eight leading bits, and again, is exact, and so is the sum), so
// that a state of 32 bits loses nothing on its way through a product.  (fp32 matrix instructions take 16 times as long as one in bf16.)
// Inner index: lane group g holds values 32 s + 4 g ... + 3 and 32 s + 16 + 4 g ... + 3, which is what it has of two accumulator tiles of
// 16 rows: what one product leaves is the next one's operand without a move.
template <int N>
struct Planes {
  u32x4 p[N];
};

template <typename T>
struct Kind;
template <>
struct Kind<unsigned short> {
  static constexpr int kIn = 1, kChunk = 64;   // planes of an operand that is given
  static constexpr int kOut = 2;               // planes of what goes into outputs of this type alone
};
template <>
struct Kind<float> {
  static constexpr int kIn = 3, kChunk = 32, kOut = 3;
};

__device__ static inline f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }

__device__ static inline f32x4 mma1(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8*>(&a), *reinterpret_cast<bf16x8*>(&b), c, 0, 0, 0);
}
// c + a b, terms below 2^-24 of the largest left out, the smallest first.  MA, MB: planes to take.
template <int MA, int MB, int NA, int NB>
__device__ static inline f32x4 mma_of(const Planes<NA>& a, const Planes<NB>& b, f32x4 c) {
  constexpr int W = MA > MB ? MA : MB;
#pragma unroll
  for (int w = W - 1; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < MA; ++i)
      if (w - i >= 0 && w - i < MB) c = mma1(a.p[i], b.p[w - i], c);
  return c;
}
template <int NA, int NB>
__device__ static inline f32x4 mma(const Planes<NA>& a, const Planes<NB>& b, f32x4 c) {
  return mma_of<NA, NB>(a, b, c);
}

// c_r + a_r b for some tiles at once, plane by plane: a product of 16 x 16 x 32 can follow another one into the same sums only after 8 of
// its cycles more than it takes, and products of other tiles fill them.
template <int MA, int MB, int R, int NA, int NB>
__device__ static inline void mma_rows(const Planes<NA> (&a)[R], const Planes<NB>& b, f32x4 (&c)[R]) {
  constexpr int W = MA > MB ? MA : MB;
#pragma unroll
  for (int w = W - 1; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < MA; ++i)
      if (w - i >= 0 && w - i < MB)
#pragma unroll
        for (int r = 0; r < R; ++r) c[r] = mma1(a[r].p[i], b.p[w - i], c[r]);
}
// c_r + a b_r
template <int MA, int MB, int R, int NA, int NB>
__device__ static inline void mma_cols(const Planes<NA>& a, const Planes<NB> (&b)[R], f32x4 (&c)[R]) {
  constexpr int W = MA > MB ? MA : MB;
#pragma unroll
  for (int w = W - 1; w >= 0; --w)
#pragma unroll
    for (int i = 0; i < MA; ++i)
      if (w - i >= 0 && w - i < MB)
#pragma unroll
        for (int r = 0; r < R; ++r) c[r] = mma1(a.p[i], b[r].p[w - i], c[r]);
}

// What follows stays behind what came before, for the compiler's scheduler.
__device__ static inline void step_end() { __builtin_amdgcn_sched_barrier(0); }
// Of the step that ends here: first `D` reads of LDS (the next step's operands), then products with `V` vector instructions behind each
// (those make the next step's operands): a wave that has its SIMD to itself overlaps them in no other way.
template <int M, int V, int D>
__device__ static inline void interleave() {
  if constexpr (D > 0) __builtin_amdgcn_sched_group_barrier(0x100, D, 0);
#pragma unroll
  for (int i = 0; i < M; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
  }
  step_end();
}

// x as N truncated planes.
template <int N>
__device__ static inline Planes<N> split(f32x4 a, f32x4 b) {
  Planes<N> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = i < 2 ? a[2 * i] : b[2 * i - 4], hi = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
#pragma unroll
    for (int p = 0; p < N; ++p) {
      o.p[p][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
      if (p + 1 < N) {
        lo -= __uint_as_float(__float_as_uint(lo) & 0xffff0000u);
        hi -= __uint_as_float(__float_as_uint(hi) & 0xffff0000u);
      }
    }
  }
  return o;
}

// 16-byte chunk q of row `row` lies at position q ^ swz<RB>(row).  Row reads fetch 8 bytes of one chunk (and its neighbour) from 16 rows,
// transposing reads two neighbouring chunks of eight rows 0 ... 7 (8 ... 15): both on distinct banks for 32 lanes.
template <int RB>
__device__ constexpr int swz(int row) {
  if (RB == 32) return 0;   // eight rows are 256 bytes by themselves
  static_assert(RB == 32 || RB == 64 || RB == 128 || RB % 256 == 0, "rows of 64, 128 or whole 256 bytes");
  if (RB == 64) return ((row >> 2) & 1) << 1;
  if (RB == 128) return ((row >> 1) & 3) << 1 | ((row >> 3) & 1);
  return (row & 7) << 1 | ((row >> 3) & 1);
}

// A tile of R rows and D columns of bf16 in LDS, N planes of it.
template <int R, int D, int N>
struct Mat {
  static constexpr int RB = 2 * D, kBytes = R * RB, kAll = N * kBytes;
  // inner values 32 s ... of row 16 r + i
  __device__ static int row_base(Lane l) { return l.i * RB + (((l.g >> 1) ^ swz<RB>(l.i)) << 4) + 8 * (l.g & 1); }
  __device__ static Planes<N> row(int tile, int base, int r, int s) {
    Planes<N> f;
    const int at = base ^ (s << 6);
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const u32x2 a = lds_get<u32x2>(tile + p * kBytes + r * 16 * RB + at), b = lds_get<u32x2>(tile + p * kBytes + r * 16 * RB + (at ^ 32));
      f.p[p] = u32x4{a[0], a[1], b[0], b[1]};
    }
    return f;
  }
  // inner values: rows 32 s ... of column 16 t + i
  __device__ static int col_base(Lane l) {
    const int r = 4 * l.g + (l.i >> 2);
    return r * RB + ((((l.i >> 1) & 1) ^ swz<RB>(r)) << 4) + 8 * (l.i & 1);
  }
  __device__ static Planes<N> col(int tile, int base, int t, int s) {
    Planes<N> f;
    const int at = tile + 32 * s * RB + (base ^ (t << 5));
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const u32x2 a = lds_get_tr16(at + p * kBytes), b = lds_get_tr16(at + p * kBytes + 16 * RB);
      f.p[p] = u32x4{a[0], a[1], b[0], b[1]};
    }
    return f;
  }
  // the values of rows 16 r + 4 g ... + 3 of column 16 t + i
  __device__ static f32x4 quad(int tile, int base, int t, int r) {
    f32x4 v = zero4();
#pragma unroll
    for (int p = N - 1; p >= 0; --p) {
      const u32x2 a = lds_get_tr16(tile + p * kBytes + 16 * r * RB + (base ^ (t << 5)));
      v += f32x4{__uint_as_float(a[0] << 16), __uint_as_float(a[0] & 0xffff0000u), __uint_as_float(a[1] << 16), __uint_as_float(a[1] & 0xffff0000u)};
    }
    return v;
  }
  // columns 16 t + 4 g ... + 3 of row 16 r + i (with row_base)
  __device__ static f32x4 row_quad(int tile, int base, int r, int t) {
    f32x4 v = zero4();
#pragma unroll
    for (int p = N - 1; p >= 0; --p) {
      const u32x2 a = lds_get<u32x2>(tile + p * kBytes + 16 * r * RB + (base ^ (t << 5)));
      v += f32x4{__uint_as_float(a[0] << 16), __uint_as_float(a[0] & 0xffff0000u), __uint_as_float(a[1] << 16), __uint_as_float(a[1] & 0xffff0000u)};
    }
    return v;
  }
  __device__ static void put_row_quad(int tile, int base, int r, int t, f32x4 v) {
    const Planes<N> f = split<N>(v, v);
#pragma unroll
    for (int p = 0; p < N; ++p) lds_put(tile + p * kBytes + 16 * r * RB + (base ^ (t << 5)), u32x2{f.p[p][0], f.p[p][1]});
  }
  // eight columns 8 q ... + 7 of a row
  __device__ static void put8(int tile, int row, int q, const Planes<N>& f) {
#pragma unroll
    for (int p = 0; p < N; ++p) lds_put(tile + p * kBytes + row * RB + ((q ^ swz<RB>(row & 15)) << 4), f.p[p]);
  }
};

__device__ static inline f32x4 as_float(u32x4 v) { return f32x4{__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3])}; }
__device__ static inline u32x4 as_bits(f32x4 v) { return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}; }

// C rows of D columns on their way from memory to LDS, eight columns a unit; zeros behind the last row and column.
// VEC: rows begin at multiples of 16 bytes and are whole 16 bytes long.
template <typename T, int C, int D, int NTH, bool VEC>
struct Load {
  static constexpr int kPer = D / 8, kUnits = C * kPer, kEach = (kUnits + NTH - 1) / NTH, kP = (int)sizeof(T) / 2;
  static constexpr int kIn = Kind<T>::kIn;
  u32x4 r[VEC ? kEach : 1][kP];
  Piece<T> p[VEC ? 1 : kEach][kP];
  unsigned odd;
  int have[VEC ? 1 : kEach];
  __device__ void load(const Rows& x, int r0, int nr, int tid) {
    unsigned skew = 0;
    const Buffer b = VEC ? x.rows(r0, nr) : x.loose(r0, nr, skew);
    odd = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int u = tid + e * NTH, row = u / kPer;
      const unsigned c = (unsigned)(u % kPer) * 8u * (unsigned)sizeof(T), at = (unsigned)row * x.row + c + skew;
      const bool there = row < nr && (kUnits % NTH == 0 || u < kUnits);
#pragma unroll
      for (int k = 0; k < kP; ++k) {
        if (VEC) r[VEC ? e : 0][k] = __builtin_amdgcn_raw_buffer_load_b128(b, there && c + 16u * k < x.width ? at + 16u * k : kNowhere, 0, 0);
        else p[VEC ? 0 : e][k].load(b, there && c + 16u * k < x.width ? at + 16u * k : kNowhere);
      }
      if (!VEC) {
        odd |= (at >> 1 & 1u) << e;
        have[VEC ? 0 : e] = there ? (int)x.width - (int)c : 0;
      }
    }
  }
  // the unit's values as planes
  __device__ Planes<kIn> get(int e) const {
    u32x4 v[kP];
#pragma unroll
    for (int k = 0; k < kP; ++k) v[k] = VEC ? r[VEC ? e : 0][k] : p[VEC ? 0 : e][k].get((odd >> e & 1u) * 16u, have[VEC ? 0 : e] - 16 * k);
    if constexpr (kIn == 1) return Planes<1>{{v[0]}};
    else return split<kIn>(as_float(v[0]), as_float(v[kP - 1]));
  }
  template <typename M>
  __device__ void store(int tile, int tid) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int u = tid + e * NTH;
      if (kUnits % NTH == 0 || u < kUnits) M::put8(tile, u / kPer, u % kPer, get(e));
    }
  }
};

// A triangle in operand order on its way from scratch memory to LDS: N planes of blocks of 64 lanes x 8 values.
template <int NB, int N, int NTH>
struct LoadTri {
  static constexpr int kUnits = N * NB * 64, kEach = (kUnits + NTH - 1) / NTH;
  u32x4 r[kEach];
  __device__ void load(const u32x4* from, int tid) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int u = tid + e * NTH;
      if (kUnits % NTH == 0 || u < kUnits) r[e] = from[u];
    }
  }
  __device__ void store(int tile, int tid) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int u = tid + e * NTH;
      if (kUnits % NTH == 0 || u < kUnits) lds_put(tile + 16 * u, r[e]);
    }
  }
};
// Waits for all memory operations of the wave but the last `N`.
template <int N>
__device__ static inline void wait_loads() {
  static_assert(N < 64, "what vmcnt counts");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
}

// The blocks of a triangle of one inner step: row tiles of a lower one from 2 s on, of an upper one up to 2 s + 1.
template <int C, bool LOWER>
struct Tri {
  static constexpr int NT = C / 16;
  __device__ static constexpr int first(int s) { return LOWER ? 2 * s : 0; }
  __device__ static constexpr int last(int s) { return LOWER ? NT - 1 : C == 32 ? 1 : 2 * s + 1; }
  __device__ static constexpr int block(int r, int s) { return C == 32 ? r : LOWER ? (r < 2 ? r : 2 * (r - 1) + s) : (r < 2 ? 2 * r + s : r + 2); }
};
// One plane of the blocks of step s.
template <int C, bool LOWER>
__device__ static inline void tri_plane(int tile, int base, int s, int plane, u32x4 (&t)[C / 16]) {
  typedef Tri<C, LOWER> X;
#pragma unroll
  for (int r = 0; r < C / 16; ++r)
    if (r >= X::first(s) && r <= X::last(s)) t[r] = lds_get<u32x4>(base + tile + (plane * blocks_of(C) + X::block(r, s)) * 1024);
}
// x_r + the blocks' products with b, plane by plane of the triangle, the smallest first (TRANS: b on the left).
template <int C, bool LOWER, bool TRANS, int MA, int MB, int N>
__device__ static inline void mma_step(const u32x4 (&t)[MA][C / 16], int s, const Planes<N>& b, f32x4 (&x)[C / 16]) {
  typedef Tri<C, LOWER> X;
#pragma unroll
  for (int i = MA - 1; i >= 0; --i)
#pragma unroll
    for (int j = (MA > MB ? MA : MB) - 1 - i; j >= 0; --j)
      if (j < MB)
#pragma unroll
        for (int r = 0; r < C / 16; ++r)
          if (r >= X::first(s) && r <= X::last(s)) x[r] = TRANS ? mma1(b.p[j], t[i][r], x[r]) : mma1(t[i][r], b.p[j], x[r]);
}

// x_r + triangle . b (or b . triangle, TRANS): plane by plane of the triangle, the smallest first; a row's two blocks into sums of their own.
template <int C, bool LOWER, bool TRANS, int MA, int MB, int NA, int NB_>
__device__ static inline void mma_tri(int tile, int base, const Planes<NB_> (&b)[C / 32], f32x4 (&x)[C / 16]) {
  constexpr int NB = blocks_of(C);
  f32x4 more[2] = {zero4(), zero4()};
#pragma unroll
  for (int i = MA - 1; i >= 0; --i) {
    u32x4 t[NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) t[k] = lds_get<u32x4>(base + tile + i * NB * 1024 + k * 1024);
#pragma unroll
    for (int j = (MA > MB ? MA : MB) - 1 - i; j >= 0; --j) {
      if (j >= MB) continue;
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        // block k: row tile r, inner step s
        const int r = C == 32 ? k : LOWER ? (k < 2 ? k : k < 4 ? 2 : 3) : (k < 4 ? k >> 1 : k - 2);
        const int s = C == 32 ? 0 : LOWER ? (k < 2 ? 0 : k & 1) : (k < 4 ? k & 1 : 1);
        const bool second = C == 64 && (LOWER ? k == 3 || k == 5 : k == 1 || k == 3);
        f32x4& y = second ? more[LOWER ? (k == 5) : (k == 3)] : x[r];
        y = TRANS ? mma1(b[s].p[j], t[k], y) : mma1(t[k], b[s].p[j], y);
      }
    }
  }
  if constexpr (C == 64) {
    x[LOWER ? 2 : 0] += more[0];
    x[LOWER ? 3 : 1] += more[1];
  }
}

// Rows of a (b,h), from column col0 on.
template <typename T>
__device__ static inline Rows rows_at(const void* x, const Args& A, int bh, int d, int n, int col0, int cols) {
  return rows_of<T>(x, bh / A.H, bh % A.H, A.H, A.L, d, A.layout, 0, n, col0, cols > 0 ? cols : 0);
}
__device__ static inline int length_of(const Args& A, int bh) { return A.lengths != nullptr ? min(max(A.lengths[bh / A.H], 0), A.L) : A.L; }
// Element of a [B, H, L] (or [B, L, H]) array of a (b,h) at token t.
__device__ static inline long long gate_at(const Args& A, int bh, int t) {
  return A.layout == DARK_BHLD ? (long long)bh * A.L + t : ((long long)(bh / A.H) * A.L + t) * A.H + bh % A.H;
}
__device__ static inline long long chunk_at(const Args& A, int bh, int c) { return (long long)bh * A.chunks + c; }

// Four values to columns c ... of a row of a tensor: `left` bytes of them exist.
template <typename T>
__device__ static inline void store_quad(char* p, int left, f32x4 v) {
  if constexpr (sizeof(T) == 2) {
    const u32x2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    if (left >= 8) {
      __builtin_memcpy(p, &w, 8);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (left > 2 * j) reinterpret_cast<unsigned short*>(p)[j] = (unsigned short)(w[j / 2] >> 16 * (j & 1));
    }
  } else {
    if (left >= 16) {
      __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (left > 4 * j) reinterpret_cast<float*>(p)[j] = v[j];
    }
  }
}
template <typename T>
__device__ static inline void buffer_quad(Buffer b, unsigned at, f32x4 v) {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}, b, at, 0, 0);
  else __builtin_amdgcn_raw_buffer_store_b128(as_bits(v), b, at, 0, 0);
}
// Zeros to the rows begin ... end - 1 of a (b,h), by `nth` threads.
template <typename T>
__device__ static inline void zero_rows(const Rows& x, int begin, int end, int tid, int nth) {
  const int cols = (int)(x.width / sizeof(T)), lane = tid & 63;
  for (int r = begin + tid / 64; r < end; r += nth / 64)
    for (int c = lane; c < cols; c += 64) reinterpret_cast<T*>(x.at(r))[c] = (T)0;
}

}  // namespace delta
}  // namespace dark
