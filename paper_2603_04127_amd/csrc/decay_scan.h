// The chunked scan of decayed linear attention and the states of its segments, for one element type (see decay.h for the mathematics).
//
// A workgroup of four waves walks the rows of a segment of one (b,h) in chunks of C rows, for a block of D2 columns of x3 and y.
// The state U [D1, D2] stays in the accumulators of the products that update it: each wave owns D2 / 4 of its columns, and what it
// owns serves the next chunk's readout as an operand without leaving the registers: an accumulator tile holds four consecutive
// rows of a column in a lane, and as the order in which a product runs over its inner dimension is free as long as both operands
// keep to it, two such tiles are one operand of 32, met by x1 rows that are read in the same order (`row_perm`).
// Per chunk: P = x1 x2^T, decayed and masked, by all waves together through LDS; y^T = U^T x1^T + x3^T P^T; U' = g^C U + x2^T (w x3).
#pragma once

#include "decay.h"

namespace dark {
namespace decay {

using namespace fz;

// 16-byte chunk q of row `row` of a tile in LDS whose rows are RB bytes long lies at position q ^ swz<RB>(row).  Rows read side by
// side (16 rows, one chunk each) and columns read by the transposing reads (four rows, two neighbouring chunks; the other half of
// the 32 lanes that the LDS serves together eight rows further on) both fall onto distinct banks: with rows of 256 bytes the four
// low bits of the row permute all 16 chunks, neighbours of four rows two chunks apart.
template <int RB>
__device__ static inline int swz(int row) {
  static_assert(RB == 128 || RB % 256 == 0, "rows of 128 or whole 256 bytes");
  if (RB == 128) return ((row >> 2) & 1) | ((row >> 1) & 1) << 1 | ((row >> 3) & 1) << 2;
  return ((row >> 2) & 1) | (row & 3) << 1 | ((row >> 3) & 1) << 3;
}
template <int RB>
__device__ static inline int at(int row, int q) { return row * RB + ((q ^ swz<RB>(row)) << 4); }

// Operands of a product over 32 values of the inner dimension: eight a lane, those of lane group g = lane / 16.
template <typename T>
struct Op;

template <>
struct Op<unsigned short> {
  typedef u32x4 frag;
  static constexpr int kPlanes = 3;
  static constexpr int kChunk = kChunkBf16;
  __device__ static f32x4 mma(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8*>(&a), *reinterpret_cast<bf16x8*>(&b), c, 0, 0, 0);
  }
  // values k0 + 8 g ... + 7 of a row
  template <int RB>
  __device__ static frag row(const char* tile, int r, int k0, int g) {
    return *reinterpret_cast<const u32x4*>(tile + at<RB>(r, k0 / 8 + g));
  }
  // values k0 + 4 g ... + 3 and k0 + 16 + 4 g ... + 3: the order of two accumulator tiles
  template <int RB>
  __device__ static frag row_perm(const char* tile, int r, int k0, int g) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(tile + at<RB>(r, k0 / 8 + (g >> 1)) + 8 * (g & 1));
    const u32x2 b = *reinterpret_cast<const u32x2*>(tile + at<RB>(r, k0 / 8 + 2 + (g >> 1)) + 8 * (g & 1));
    return frag{a[0], a[1], b[0], b[1]};
  }
  // rows r0 + 8 g ... + 7 of column c0 + lane % 16
  template <int RB>
  __device__ static frag col(const char* tile, int r0, int c0, int lane) {
    const int i = lane & 15, r = r0 + 8 * (lane >> 4) + (i >> 2), q = c0 / 8 + ((i >> 1) & 1);
    const u32x2 a = lds_read_tr16(reinterpret_cast<const unsigned short*>(tile + at<RB>(r, q) + 8 * (i & 1)));
    const u32x2 b = lds_read_tr16(reinterpret_cast<const unsigned short*>(tile + at<RB>(r + 4, q) + 8 * (i & 1)));
    return frag{a[0], a[1], b[0], b[1]};
  }
  // Two accumulator tiles as an operand.  Rounded to bf16 once (2^-8 relative): the product goes into an output of that type.
  __device__ static frag state(f32x4 a, f32x4 b) {
    return frag{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])};
  }
  // w x as the sum of three bf16 operands: the state is a 32-bit result, so its terms keep their 24 bits (8 + 8 + 8).
  __device__ static void weighted(frag x, const float* w, frag* out) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo = __uint_as_float(x[i] << 16) * w[2 * i], hi = __uint_as_float(x[i] & 0xffff0000u) * w[2 * i + 1];
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) {
        const unsigned u = pack_bf16(lo, hi);
        out[p][i] = u;
        lo -= __uint_as_float(u << 16);
        hi -= __uint_as_float(u & 0xffff0000u);
      }
    }
  }
  // four values of P, columns c ... c + 3 of row r
  template <int RB>
  __device__ static void put4(char* tile, int r, int c, f32x4 v) {
    *reinterpret_cast<u32x2*>(tile + at<RB>(r, c / 8) + 2 * (c & 7)) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
  __device__ static void store4(unsigned short* p, f32x4 v) {
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
  __device__ static void store1(unsigned short* p, float v) { *p = (unsigned short)pack_bf16(v, 0.f); }
};

template <>
struct Op<float> {
  struct frag {
    f32x4 v[2];
  };
  static constexpr int kPlanes = 1;
  static constexpr int kChunk = kChunkF32;
  // eight products over four values each; the lane group's value j of both operands makes the inner index
  __device__ static f32x4 mma(const frag& a, const frag& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j >> 2][j & 3], b.v[j >> 2][j & 3], c, 0, 0, 0);
    return c;
  }
  template <int RB>
  __device__ static frag row(const char* tile, int r, int k0, int g) {
    return frag{{*reinterpret_cast<const f32x4*>(tile + at<RB>(r, k0 / 4 + 2 * g)),
                 *reinterpret_cast<const f32x4*>(tile + at<RB>(r, k0 / 4 + 2 * g + 1))}};
  }
  template <int RB>
  __device__ static frag row_perm(const char* tile, int r, int k0, int g) {
    return frag{{*reinterpret_cast<const f32x4*>(tile + at<RB>(r, k0 / 4 + g)),
                 *reinterpret_cast<const f32x4*>(tile + at<RB>(r, k0 / 4 + 4 + g))}};
  }
  template <int RB>
  __device__ static frag col(const char* tile, int r0, int c0, int lane) {
    frag f;
    const int i = lane & 15, r = r0 + 8 * (lane >> 4);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      f.v[j >> 2][j & 3] = *reinterpret_cast<const float*>(tile + at<RB>(r + j, c0 / 4 + (i >> 2)) + 4 * (i & 3));
    return f;
  }
  __device__ static frag state(f32x4 a, f32x4 b) { return frag{{a, b}}; }
  __device__ static void weighted(const frag& x, const float* w, frag* out) {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[0].v[j >> 2][j & 3] = x.v[j >> 2][j & 3] * w[j];
  }
  template <int RB>
  __device__ static void put4(char* tile, int r, int c, f32x4 v) {
    *reinterpret_cast<f32x4*>(tile + at<RB>(r, c / 4)) = v;
  }
  __device__ static void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
  __device__ static void store1(float* p, float v) { *p = v; }
};

// Where the rows of a (b,h) lie: row r is token r, or counted from the end token n - 1 - r.
template <typename T>
struct Rows {
  const T* base;
  long long stride;   // elements from one row to the next (negative: counted from the end)
};
template <typename T>
__device__ static inline Rows<T> rows_of(const void* x, int b, int h, int H, int L, int d, int layout, int reverse, int n) {
  const long long stride = layout == DARK_BHLD ? d : (long long)H * d;
  const T* base = static_cast<const T*>(x) + (layout == DARK_BHLD ? ((long long)b * H + h) * L * d : ((long long)b * L * H + h) * d);
  if (!reverse) return {base, stride};
  return {base + (n > 0 ? (n - 1) * stride : 0), -stride};
}

// A tile of C rows and D columns on its way to LDS: NCH = C D sizeof(T) / 16 / 256 pieces of 16 bytes a thread, zeros behind the last
// row and column (what lies there in memory is never read).  VEC: rows begin at multiples of 16 bytes and are whole pieces long.
template <typename T, int C, int D, bool VEC>
struct Tile {
  static constexpr int kPieces = D * (int)sizeof(T) / 16;   // of a row
  static constexpr int kEach = C * kPieces / 256;
  static constexpr int kPer = 16 / (int)sizeof(T);
  static_assert(C * kPieces % 256 == 0, "whole pieces a thread");
  u32x4 r[kEach];
  __device__ void load(Rows<T> x, int r0, int nr, int col0, int d, int tid) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = tid + 256 * i, row = e / kPieces, c = col0 + (e % kPieces) * kPer;
      r[i] = u32x4{0, 0, 0, 0};
      if (row >= nr || c >= d) continue;
      const T* p = x.base + (long long)(r0 + row) * x.stride + c;
      if (VEC) {
        r[i] = *reinterpret_cast<const u32x4*>(p);
      } else {
        T v[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[j] = c + j < d ? p[j] : (T)0;
        __builtin_memcpy(&r[i], v, 16);
      }
    }
  }
  __device__ void store(char* tile, int tid) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = tid + 256 * i;
      *reinterpret_cast<u32x4*>(tile + at<D * (int)sizeof(T)>(e / kPieces, e % kPieces)) = r[i];
    }
  }
};

// The decay in the log2 domain.  exp(-inf) = 0 as a large negative number, so that 0 * -inf does not arise: g^0 = 1.
__device__ static inline float decay_log2(const float* log_decay, int h) { return fmaxf(log_decay[h] * kLog2e, -1e30f); }
__device__ static inline float power(float a2, int n) { return fast_exp2(a2 * (float)n); }

// Weights g^(nr-1-key+off) su of the lane's keys; 0 behind the last row.
template <int KS>
__device__ static inline void key_weights(float (&w)[KS][8], float a2, int nr, int off, float su, int g) {
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = nr - 1 - (32 * ks + 8 * g + j);
      w[ks][j] = n >= 0 ? su * power(a2, n + off) : 0.f;
    }
}

// U <- g^nr U + x2^T (w x3): the columns of U that the wave owns.
template <typename T, int C, int D1, int D2, int NT>
__device__ static inline void update(f32x4 (&U)[D1 / 16][NT], const char* t2, const char* t3, const float (&w)[C / 32][8], float gn, int wave, int lane) {
  typedef Op<T> O;
#pragma unroll
  for (int kt = 0; kt < D1 / 16; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) U[kt][nt] *= gn;
#pragma unroll
  for (int ks = 0; ks < C / 32; ++ks) {
    typename O::frag x[NT][O::kPlanes];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      O::weighted(O::template col<D2 * (int)sizeof(T)>(t3, 32 * ks, 16 * (wave * NT + nt), lane), w[ks], x[nt]);
#pragma unroll
    for (int kt = 0; kt < D1 / 16; ++kt) {
      const typename O::frag k = O::template col<D1 * (int)sizeof(T)>(t2, 32 * ks, 16 * kt, lane);
#pragma unroll
      for (int p = O::kPlanes - 1; p >= 0; --p)   // the smallest terms first
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) U[kt][nt] = O::mma(k, x[nt][p], U[kt][nt]);
    }
  }
}

template <typename T, int D1, int D2>
constexpr int scan_lds() { return Op<T>::kChunk * (2 * D1 + D2 + Op<T>::kChunk) * (int)sizeof(T); }
template <typename T, int D1, int D2>
constexpr int state_lds() { return Op<T>::kChunk * (D1 + D2) * (int)sizeof(T); }

template <typename T, int D1, int D2, bool VEC>
__global__ __launch_bounds__(256) void k_decay_scan(Scans A) {
  typedef Op<T> O;
  constexpr int C = O::kChunk, QT = C / 16, KS = C / 32, NT = D2 / 64, KT = D1 / 16, K1 = D1 / 32;
  constexpr int RB1 = D1 * (int)sizeof(T), RB2 = D2 * (int)sizeof(T), RBP = C * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(256))) char smem[];
  char* const t1 = smem;
  char* const t2 = t1 + C * RB1;
  char* const t3 = t2 + C * RB1;
  char* const tp = t3 + C * RB2;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l15 = lane & 15, g = lane >> 4;
  Scan a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  if (blockIdx.z == 2) a = A.s[2];
  const int bh = blockIdx.x / A.nseg, seg = blockIdx.x % A.nseg, b = bh / A.H, h = bh % A.H, col0 = blockIdx.y * D2;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const float a2 = decay_log2(A.log_decay, h);
  const int begin = seg * A.seg_len, end = min(begin + A.seg_len, A.L);
  T* const ybase = const_cast<T*>(rows_of<T>(a.y, b, h, A.H, A.L, a.d2, A.layout, 0, n).base);
  const long long ystride = A.layout == DARK_BHLD ? a.d2 : (long long)A.H * a.d2;
  // rows behind the sequence
  for (int r = a.y != nullptr ? max(begin, n) + (tid >> 6) : end; r < end; r += 4)
    for (int c = col0 + lane; c < min(col0 + D2, a.d2); c += 64) ybase[r * ystride + c] = (T)0;
  if (begin >= n && seg > 0) return;   // segment 0 passes the state on even when there are no rows

  const Rows<T> x1 = rows_of<T>(a.x1, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n);
  const Rows<T> x2 = rows_of<T>(a.x2, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n);
  const Rows<T> x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n);
  const int last = min(end, n);
  Tile<T, C, D1, VEC> p1, p2;
  Tile<T, C, D2, VEC> p3;
  p1.load(x1, begin, last - begin, 0, a.d1, tid);
  p2.load(x2, begin, last - begin, 0, a.d1, tid);
  p3.load(x3, begin, last - begin, col0, a.d2, tid);

  // the state: rows 16 kt + 4 g ... + 3 of column col0 + 16 (wave NT + nt) + lane % 16
  f32x4 U[KT][NT];
  const long long uat = A.nseg > 1 ? (long long)bh * A.nseg + seg : bh;
  const float* const uin = a.u_in != nullptr ? a.u_in + uat * a.d1 * a.d2 : nullptr;
  bool carried = uin != nullptr;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * kt + 4 * g, c = col0 + 16 * (wave * NT + nt) + l15;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        U[kt][nt][j] = carried && row + j < a.d1 && c < a.d2 ? uin[a.transposed ? (long long)c * a.d1 + row + j : (long long)(row + j) * a.d2 + c] : 0.f;
    }
  // Tiles of P above the diagonal that a product over 32 keys reads: zero from here on, never written again.
  for (int e = tid; e < C * RBP / 16; e += 256) *reinterpret_cast<u32x4*>(tp + 16 * e) = u32x4{0, 0, 0, 0};

  float w[KS][8];
  key_weights<KS>(w, a2, C, a.off, a.su, g);
  float lead[QT];   // sr g^(r+1-off) of the lane's rows
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) lead[qt] = a.sr * power(a2, 16 * qt + l15 + 1 - a.off);
  float gn = power(a2, C);

  for (int r0 = begin; r0 < last; r0 += C) {
    const int nr = min(C, last - r0);
    lds_barrier();   // the tiles' readers are done
    p1.store(t1, tid);
    p2.store(t2, tid);
    p3.store(t3, tid);
    lds_barrier();
    if (r0 + C < last) {
      p1.load(x1, r0 + C, last - r0 - C, 0, a.d1, tid);
      p2.load(x2, r0 + C, last - r0 - C, 0, a.d1, tid);
      p3.load(x3, r0 + C, last - r0 - C, col0, a.d2, tid);
    }
    // P: the tiles on and below the diagonal, dealt out to the waves
#pragma unroll
    for (int i = 0; i < (QT * (QT + 1) / 2 + 3) / 4; ++i) {
      const int t = wave + 4 * i;
      if (t < QT * (QT + 1) / 2) {
        const int qt = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, kt = t - qt * (qt + 1) / 2;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K1; ++k)
          s = O::mma(O::template row<RB1>(t2, 16 * kt + l15, 32 * k, g), O::template row<RB1>(t1, 16 * qt + l15, 32 * k, g), s);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int apart = 16 * (qt - kt) + l15 - 4 * g - j;
          s[j] = apart >= 0 ? s[j] * (a.sp * power(a2, max(apart, 0))) : 0.f;
        }
        O::template put4<RBP>(tp, 16 * qt + l15, 16 * kt + 4 * g, s);
      }
    }
    f32x4 y[NT][QT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) y[nt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (carried) {
#pragma unroll
      for (int k = 0; k < K1; ++k) {
        typename O::frag u[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) u[nt] = O::state(U[2 * k][nt], U[2 * k + 1][nt]);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const typename O::frag x = O::template row_perm<RB1>(t1, 16 * qt + l15, 32 * k, g);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) y[nt][qt] = O::mma(u[nt], x, y[nt][qt]);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) y[nt][qt] *= lead[qt];
    }
    lds_barrier();   // P is there
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      typename O::frag v[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) v[nt] = O::template col<RB2>(t3, 32 * ks, 16 * (wave * NT + nt), lane);
#pragma unroll
      for (int qt = 2 * ks; qt < QT; ++qt) {
        const typename O::frag p = O::template row<RBP>(tp, 16 * qt + l15, 32 * ks, g);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) y[nt][qt] = O::mma(v[nt], p, y[nt][qt]);
      }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = r0 + 16 * qt + l15;
      if (r < last && a.y != nullptr) {
        T* const row = ybase + (a.reverse ? n - 1 - r : r) * ystride;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int c = col0 + 16 * (wave * NT + nt) + 4 * g;
          if (VEC) {
            if (c < a.d2) O::store4(row + c, y[nt][qt]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c + j < a.d2) O::store1(row + c + j, y[nt][qt][j]);
          }
        }
      }
    }
    if (r0 + C < last || (last == n && a.u_out != nullptr)) {
      if (nr < C) {
        key_weights<KS>(w, a2, nr, a.off, a.su, g);
        gn = power(a2, nr);
      }
      update<T, C, D1, D2, NT>(U, t2, t3, w, gn, wave, lane);
      carried = true;
    }
  }
  if (last != n || a.u_out == nullptr) return;
  float* const uo = a.u_out + (long long)bh * a.d1 * a.d2;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * kt + 4 * g, c = col0 + 16 * (wave * NT + nt) + l15;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (row + j < a.d1 && c < a.d2) uo[a.transposed ? (long long)c * a.d1 + row + j : (long long)(row + j) * a.d2 + c] = U[kt][nt][j];
    }
}

template <typename T, int D1, int D2, bool VEC>
__global__ __launch_bounds__(256) void k_decay_state(States A) {
  typedef Op<T> O;
  constexpr int C = O::kChunk, KS = C / 32, NT = D2 / 64, KT = D1 / 16;
  extern __shared__ __attribute__((aligned(256))) char smem[];
  char* const t2 = smem;
  char* const t3 = t2 + C * D1 * (int)sizeof(T);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l15 = lane & 15, g = lane >> 4;
  State a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  const int segs = A.nseg - 1, bh = blockIdx.x / segs, seg = blockIdx.x % segs, b = bh / A.H, h = bh % A.H, col0 = blockIdx.y * D2;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const int begin = seg * A.seg_len, end = begin + A.seg_len;
  if (end >= n) return;   // nothing follows
  const float a2 = decay_log2(A.log_decay, h);
  const Rows<T> x2 = rows_of<T>(a.x2, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n);
  const Rows<T> x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n);
  Tile<T, C, D1, VEC> p2;
  Tile<T, C, D2, VEC> p3;
  p2.load(x2, begin, C, 0, a.d1, tid);
  p3.load(x3, begin, C, col0, a.d2, tid);
  f32x4 U[KT][NT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) U[kt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float w[KS][8];
  key_weights<KS>(w, a2, C, a.off, a.su, g);
  const float gn = power(a2, C);
  for (int r0 = begin; r0 < end; r0 += C) {
    lds_barrier();
    p2.store(t2, tid);
    p3.store(t3, tid);
    lds_barrier();
    if (r0 + C < end) {
      p2.load(x2, r0 + C, C, 0, a.d1, tid);
      p3.load(x3, r0 + C, C, col0, a.d2, tid);
    }
    update<T, C, D1, D2, NT>(U, t2, t3, w, gn, wave, lane);
  }
  float* const uo = a.seg + ((long long)bh * A.nseg + seg) * a.d1 * a.d2;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * kt + 4 * g, c = col0 + 16 * (wave * NT + nt) + l15;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (row + j < a.d1 && c < a.d2) uo[(long long)(row + j) * a.d2 + c] = U[kt][nt][j];
    }
}

template <typename T, int D1, int D2, bool VEC>
static dark_status launch_scan(const Scans& a, int n, hipStream_t st) {
  constexpr int lds = scan_lds<T, D1, D2>();
  DARK_TRY(allow_lds(k_decay_scan<T, D1, D2, VEC>, lds));
  const dim3 grid((unsigned)((long long)a.B * a.H * a.nseg), (unsigned)((a.s[0].d2 + D2 - 1) / D2), (unsigned)n);
  DARK_LAUNCH(KID_DECAY_SCAN, st, (k_decay_scan<T, D1, D2, VEC>), grid, dim3(256), lds, a);
  return DARK_OK;
}
template <typename T, int D1, int D2, bool VEC>
static dark_status launch_state(const States& a, int n, hipStream_t st) {
  constexpr int lds = state_lds<T, D1, D2>();
  DARK_TRY(allow_lds(k_decay_state<T, D1, D2, VEC>, lds));
  const dim3 grid((unsigned)((long long)a.B * a.H * (a.nseg - 1)), (unsigned)((a.s[0].d2 + D2 - 1) / D2), (unsigned)n);
  DARK_LAUNCH(KID_DECAY_STATE, st, (k_decay_state<T, D1, D2, VEC>), grid, dim3(256), lds, a);
  return DARK_OK;
}

// The instance that holds d1 inner values, with 64 columns a workgroup where x3 has no more (or the state of 256 x 128 would take
// half of the registers), else 128.
#define DARK_DECAY_PICK(what, T, a, n, st)                                                                  \
  do {                                                                                                      \
    const int d1 = (a).s[0].d1, d2 = (a).s[0].d2;                                                           \
    const bool vec = d1 * (int)sizeof(T) % 16 == 0 && d2 * (int)sizeof(T) % 16 == 0;                        \
    if (d1 <= 64 && d2 <= 64) return vec ? what<T, 64, 64, true>(a, n, st) : what<T, 64, 64, false>(a, n, st);      \
    if (d1 <= 64) return vec ? what<T, 64, 128, true>(a, n, st) : what<T, 64, 128, false>(a, n, st);        \
    if (d1 <= 128 && d2 <= 64) return vec ? what<T, 128, 64, true>(a, n, st) : what<T, 128, 64, false>(a, n, st);   \
    if (d1 <= 128) return vec ? what<T, 128, 128, true>(a, n, st) : what<T, 128, 128, false>(a, n, st);     \
    return vec ? what<T, 256, 64, true>(a, n, st) : what<T, 256, 64, false>(a, n, st);                      \
  } while (0)

}  // namespace decay
}  // namespace dark
