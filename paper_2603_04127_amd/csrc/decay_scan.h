// The chunked scan of decayed linear attention and the states of its segments, for one element type (see decay.h for the mathematics).
//
// A workgroup of D2 / 16 waves walks the rows of a segment of one (b,h) in chunks of C rows, for a block of D2 columns of x3 and y.
// The state U [D1, D2] stays in the accumulators of the products that update it: each wave owns 16 of its columns, and what it
// owns serves the next chunk's readout as an operand without a way through LDS: an accumulator tile holds rows 4 g ... + 3 of a column in
// lane group g, an operand of two such tiles wants rows 8 g ... + 7, and two exchanges between the lane groups make one of the other.
// With 256 rows a wave owns half of them, and the halves' readouts are joined through LDS: twice the waves on a CU whose LDS holds no
// second workgroup (24 heads of 2048 x 256, values 64 wide: 48.6 -> 43 us).
// Per chunk: P = x1 x2^T, decayed and masked, by all waves together through LDS; y^T = U^T x1^T + x3^T P^T; U' = g^C U + x2^T (w x3).
// The next chunk's rows are on their way into registers meanwhile.
// Long sequences of many heads are bound by memory: 64 heads of 8192 x 128 in 8 segments, the segment states 264 MB in 70 us (59 at least), the
// scan 575 MB in 143 us (118), 4 to 4.9 TB/s where a copy has 4.9.  With 64 wide heads (24 of 4096: states 10, scan 18 us for 28 and 55 MB; of
// the backward pass 13 and 33 us for 47 and 130 MB) memory takes over half of the time, the waits between a chunk's steps the rest; fp32
// (36 heads of 509 x 64: 7 and 12 us) waits for its products, 1.7 us of the 2.8 of a chunk.
#pragma once

#include "decay.h"
#include "rows.h"

namespace dark {
namespace decay {

using namespace fz;
using namespace rows;

// 16-byte chunk q of row `row` of a tile in LDS whose rows are RB bytes long lies at position q ^ swz<RB>(row).  The LDS serves a
// 16-byte read of rows (lane l: row l % 16, chunk l / 16) in groups of lanes {0-3, 12-15, 20-27} and {4-11, 16-19, 28-31}: rows
// 0-3 and 12-15 of one chunk together with rows 4-11 of its neighbour, and the other way round.  The transposing reads fetch two
// neighbouring chunks of four rows r ... r + 3 and of r + 8 ... r + 11 together.  Both fall onto distinct banks if the position's lowest
// bit is free within each of the two row sets, that is if bit 2 ^ bit 3 of the row lies above it, and the bits above it tell the
// eight rows of a transposing read apart.  (With bit 3 alone there, the former two-way: a third of the LDS's busy cycles.)
// The mapping is linear over xor, so that constants of a tile's position are one xor with a lane's base.
template <int RB>
__device__ constexpr int swz(int row) {
  static_assert(RB == 128 || RB % 256 == 0, "rows of 128 or whole 256 bytes");
  if (RB == 128) return ((row >> 2) & 1) | ((row >> 1) & 1) << 1 | (((row >> 3) ^ (row >> 2)) & 1) << 2;
  return ((row >> 2) & 1) | (row & 3) << 1 | (((row >> 3) ^ (row >> 2)) & 1) << 3;
}

// a: values of rows 4 g ... of a tile in lane group g, b: those of the tile below it.  Afterwards lane group g has rows 8 g ... in a
// and 8 g + 4 ... in b (of the 32).
__device__ static inline void spread(unsigned& a, unsigned& b) {
  const auto h = __builtin_amdgcn_permlane32_swap(a, b, false, false);      // {a0, a1, b0, b1}, {a2, a3, b2, b3}
  const auto q = __builtin_amdgcn_permlane16_swap(h[0], h[1], false, false);   // {a0, a2, b0, b2}, {a1, a3, b1, b3}
  a = q[0];
  b = q[1];
}

// Operands of a product over 32 values of the inner dimension: eight a lane, those of lane group g.
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
  // values 32 k + 8 g ... + 7 of row i of 16
  template <int RB>
  __device__ static int row_base(Lane l) { return l.i * RB + ((l.g ^ swz<RB>(l.i)) << 4); }
  __device__ static frag row(int tile, int base, int k) { return lds_get<u32x4>(tile + (base ^ (k << 6))); }
  // rows 8 g ... + 7 (of 32) of column 16 t + i: the lane points at row 8 g + i / 4 (+ 4), columns 16 t + 4 (i % 4) ... + 3
  template <int RB>
  __device__ static int col_base(Lane l) {
    const int r = 8 * l.g + (l.i >> 2);
    return r * RB + ((((l.i >> 1) & 1) ^ swz<RB>(r)) << 4) + 8 * (l.i & 1);
  }
  template <int RB>
  __device__ static frag col(int tile, int base, int t) {
    const u32x2 a = lds_get_tr16(tile + (base ^ (t << 5))), b = lds_get_tr16(tile + 4 * RB + (base ^ (t << 5) ^ (swz<RB>(4) << 4)));
    return frag{a[0], a[1], b[0], b[1]};
  }
  // Two accumulator tiles as an operand.  Rounded to bf16 once (2^-8 relative): the product goes into an output of that type.
  __device__ static frag state(f32x4 a, f32x4 b) {
    unsigned a0 = pack_bf16(a[0], a[1]), a1 = pack_bf16(a[2], a[3]), b0 = pack_bf16(b[0], b[1]), b1 = pack_bf16(b[2], b[3]);
    spread(a0, b0);
    spread(a1, b1);
    return frag{a0, a1, b0, b1};
  }
  // w x as the sum of three bf16 operands: a state is a 32-bit result, so its terms keep their 24 bits.  Cut off, not rounded: what is left
  // behind eight leading bits, and again behind the next eight, is exact, and so is the sum of the three.  (Two of them for a state that
  // only goes into outputs of 8 bits: calls without a wanted state 3 to 10 % shorter, backward of 24 heads of 4096 x 64 47 -> 44 us, but with
  // other outputs than beside one.)
  __device__ static void weighted(frag x, f32x4 w0, f32x4 w1, frag* out) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 w = i < 2 ? w0 : w1;
      float lo = __uint_as_float(x[i] << 16) * w[2 * (i & 1)], hi = __uint_as_float(x[i] & 0xffff0000u) * w[2 * (i & 1) + 1];
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) {
        out[p][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        lo -= __uint_as_float(__float_as_uint(lo) & 0xffff0000u);
        hi -= __uint_as_float(__float_as_uint(hi) & 0xffff0000u);
      }
    }
  }
  // four values of P: columns 16 kt + 4 g ... + 3 of row i
  template <int RB>
  __device__ static int put_base(Lane l) { return l.i * RB + (((l.g >> 1) ^ swz<RB>(l.i)) << 4) + 8 * (l.g & 1); }
  __device__ static void put4(int tile, int base, int kt, f32x4 v) {
    lds_put(tile + (base ^ (kt << 5)), u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
  }
  __device__ static void store4(__amdgpu_buffer_rsrc_t b, unsigned at, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}, b, at, 0, 0);
  }
  // to an address of any alignment; the first `left` bytes
  __device__ static void store_loose(char* p, int left, f32x4 v) {
    const u32x2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    if (left >= 8) {
      __builtin_memcpy(p, &w, 8);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (left > 2 * j) reinterpret_cast<unsigned short*>(p)[j] = (unsigned short)(w[j / 2] >> 16 * (j & 1));
    }
  }
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
  __device__ static int row_base(Lane l) { return l.i * RB + (((2 * l.g) ^ swz<RB>(l.i)) << 4); }
  __device__ static frag row(int tile, int base, int k) {
    return frag{{lds_get<f32x4>(tile + (base ^ (k << 7))), lds_get<f32x4>(tile + (base ^ (k << 7) ^ 16))}};
  }
  template <int RB>
  __device__ static int col_base(Lane l) { return 8 * l.g * RB + (((l.i >> 2) ^ swz<RB>(8 * l.g)) << 4) + 4 * (l.i & 3); }
  template <int RB>
  __device__ static frag col(int tile, int base, int t) {
    frag f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = lds_get<float>(tile + j * RB + (base ^ (t << 6) ^ (swz<RB>(j) << 4)));
    return f;
  }
  __device__ static frag state(f32x4 a, f32x4 b) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      unsigned x = __float_as_uint(a[j]), y = __float_as_uint(b[j]);
      spread(x, y);
      a[j] = __uint_as_float(x);
      b[j] = __uint_as_float(y);
    }
    return frag{{a, b}};
  }
  __device__ static void weighted(const frag& x, f32x4 w0, f32x4 w1, frag* out) {
    out[0].v[0] = x.v[0] * w0;
    out[0].v[1] = x.v[1] * w1;
  }
  template <int RB>
  __device__ static int put_base(Lane l) { return l.i * RB + ((l.g ^ swz<RB>(l.i)) << 4); }
  __device__ static void put4(int tile, int base, int kt, f32x4 v) { lds_put(tile + (base ^ (kt << 6)), v); }
  __device__ static void store4(__amdgpu_buffer_rsrc_t b, unsigned at, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, b, at, 0, 0);
  }
  __device__ static void store_loose(char* p, int left, f32x4 v) {
    if (left >= 16) {
      __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (left > 4 * j) reinterpret_cast<float*>(p)[j] = v[j];
    }
  }
};

// A tile of C rows and D columns on its way to LDS: some pieces of 16 bytes for each of NTH threads, zeros behind the last
// row and column (whatever lies there in memory).  VEC: rows begin at multiples of 16 bytes and are whole pieces long.
template <typename T, int C, int D, int NTH, bool VEC>
struct Tile {
  static constexpr int kPieces = D * (int)sizeof(T) / 16;   // of a row
  static constexpr int kEach = C * kPieces / NTH;
  static constexpr int kStep = NTH / kPieces;               // rows from one piece of a thread to its next
  static constexpr int kPer = 16 / (int)sizeof(T);
  static constexpr int RB = D * (int)sizeof(T);
  static_assert(C * kPieces % NTH == 0 && NTH % kPieces == 0 && (kStep & (kStep - 1)) == 0, "whole pieces a thread");
  u32x4 r[VEC ? kEach : 1];
  Piece<T> p[VEC ? 1 : kEach];
  unsigned odd;   // pieces that begin in the middle of a word, a bit each
  int have;
  __device__ void load(const Rows& x, int r0, int nr, int tid) {
    const unsigned c = (unsigned)(tid % kPieces) * 16u, row = x.offset(tid / kPieces, nr);
    if (VEC) {
      const Buffer b = x.rows(r0, nr);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const unsigned at = row + (unsigned)x.step(i * kStep);   // wraps around to far behind the extent where rows are counted from the end
        r[i] = __builtin_amdgcn_raw_buffer_load_b128(b, c < x.width ? at + c : kNowhere, 0, 0);
      }
    } else {
      unsigned skew;
      const Buffer b = x.loose(r0, nr, skew);
      have = (int)x.width - (int)c;
      odd = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const unsigned at = row + (unsigned)x.step(i * kStep) + c + skew;
        p[i].load(b, have > 0 && tid / kPieces + i * kStep < nr ? at : kNowhere);
        odd |= (at >> 1 & 1u) << i;
      }
    }
  }
  __device__ void store(int tile, int tid) const {
    const int row0 = tid / kPieces, base = row0 * RB + (((tid % kPieces) ^ swz<RB>(row0)) << 4);
    // kStep is a power of two and row0 below it: further rows are one xor with a constant away
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      lds_put(tile + i * kStep * RB + (base ^ (swz<RB>((i * kStep) & 15) << 4)), VEC ? r[VEC ? i : 0] : p[VEC ? 0 : i].get((odd >> i & 1u) * 16u, have));
  }
};

// The decay in the log2 domain.  exp(-inf) = 0 as a large negative number, so that 0 * -inf does not arise: g^0 = 1.
__device__ static inline float decay_log2(const float* log_decay, int h) { return fmaxf(log_decay[h] * kLog2e, -1e30f); }
__device__ static inline float power(float a2, int n) { return fast_exp2(a2 * (float)n); }

// Weights su g^(nr-1-key+off) of the chunk's keys, 0 behind the last row: C floats in LDS.
template <int C>
__device__ static inline void put_weights(int tw, float a2, int nr, int off, float su, int tid) {
  if (tid < C) lds_put(tw + 4 * tid, tid < nr ? su * power(a2, max(nr - 1 - tid, 0) + off) : 0.f);
}

// U <- U + x2^T (f w x3): the 16 columns of U that the wave owns, of its half of the rows.
template <typename T, int C, int D1, int D2, int H = 1>
__device__ static inline void update(f32x4 (&U)[D1 / 16 / H], int t2, int t3, int tw, float f, int wave, Lane l, int half = 0) {
  typedef Op<T> O;
  constexpr int RB1 = D1 * (int)sizeof(T), RB2 = D2 * (int)sizeof(T);
  const int b2 = O::template col_base<RB1>(l) ^ (half * (RB1 / H)), b3 = O::template col_base<RB2>(l);
#pragma unroll
  for (int ks = 0; ks < C / 32; ++ks) {
    typename O::frag x[O::kPlanes];
    const f32x4 w0 = f * lds_get<f32x4>(tw + 128 * ks + 32 * l.g), w1 = f * lds_get<f32x4>(tw + 128 * ks + 32 * l.g + 16);
    O::weighted(O::template col<RB2>(t3 + 32 * ks * RB2, b3, wave), w0, w1, x);
#pragma unroll
    for (int k0 = 0; k0 < D1 / 16 / H; k0 += 4) {   // four sums at a time: a product does not wait for the one before it
      typename O::frag k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = O::template col<RB1>(t2 + 32 * ks * RB1, b2, k0 + i);
#pragma unroll
      for (int p = O::kPlanes - 1; p >= 0; --p)   // the smallest terms first
#pragma unroll
        for (int i = 0; i < 4; ++i) U[k0 + i] = O::mma(k[i], x[p], U[k0 + i]);
      hold();
    }
  }
}

constexpr int halves(int d1) { return d1 == 256 ? 2 : 1; }
template <typename T, int D1, int D2>
constexpr int scan_lds() {
  return Op<T>::kChunk * ((2 * D1 + D2 + Op<T>::kChunk) * (int)sizeof(T) + 12) + 64 + (halves(D1) == 2 ? Op<T>::kChunk * D2 * 4 : 0);
}
template <typename T, int D1, int D2>
constexpr int state_lds() { return Op<T>::kChunk * ((D1 + D2) * (int)sizeof(T) + 4); }

// Waves a SIMD that the registers have to leave room for: as many as the LDS takes workgroups.
constexpr int scan_waves(int d1, int d2) { return d1 == 256 ? 2 : d1 == 128 && d2 == 64 ? 3 : 4; }
constexpr int state_waves(int d1) { return d1 == 256 ? 2 : 4; }

// The lane index anew: what is derived from it is computed where it is used, instead of held in registers all along.  Up to 64 inner
// values there are registers for it (vector instructions of a chunk 288 -> 217, the backward pass of 24 heads of 4096 x 64 47.9 -> 46.5 us).
template <int D1>
__device__ static inline Lane fresh(int lane) {
  if (D1 > 64) asm volatile("" : "+v"(lane));
  return {lane & 15, lane >> 4};
}

template <typename T, int D1, int D2, bool VEC>
__global__ __launch_bounds__(4 * D2 * halves(D1), scan_waves(D1, D2)) void k_decay_scan(Scans A) {
  typedef Op<T> O;
  constexpr int H = halves(D1), C = O::kChunk, QT = C / 16, KS = C / 32, KT = D1 / 16 / H, K1 = D1 / 32, W = H * D2 / 16, NTH = 64 * W;
  constexpr int RB1 = D1 * (int)sizeof(T), RB2 = D2 * (int)sizeof(T), RBP = C * (int)sizeof(T);
  constexpr int t1 = 0, t2 = t1 + C * RB1, t3 = t2 + C * RB1, tp = t3 + C * RB2, tw = tp + C * RBP;
  constexpr int tl = tw + 4 * C;   // sr g^(r+1-off) of the chunk's rows
  constexpr int td = tl + 4 * C;   // sp g^(n - 15), n = 0 ... C + 14 (what stands before g^0 is not used)
  constexpr int te = td + 4 * C + 64;   // readouts of the other half
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int part = wave % (D2 / 16), half = H == 2 ? wave / (D2 / 16) : 0;   // the wave's columns and rows of the state
  Scan a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  if (blockIdx.z == 2) a = A.s[2];
  const int bh = blockIdx.x / A.nseg, seg = blockIdx.x % A.nseg, b = bh / A.H, h = bh % A.H, col0 = blockIdx.y * D2;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const float a2 = decay_log2(A.log_decay, h);
  const int begin = seg * A.seg_len, end = min(begin + A.seg_len, A.L), cols = min(a.d2 - col0, D2);
  if (cols <= 0) return;   // a narrower scan than another one of the launch
  // rows behind the sequence
  if (a.y != nullptr && end > n) {
    const Rows y = rows_of<T>(a.y, b, h, A.H, A.L, a.d2, A.layout, 0, n, col0, cols);
    for (int r = max(begin, n) + wave; r < end; r += W)
      for (int c = lane; c < cols; c += 64) reinterpret_cast<T*>(const_cast<char*>(y.head) + (long long)r * y.row)[c] = (T)0;
  }
  if (begin >= n && seg > 0) return;   // segment 0 passes the state on even when there are no rows
  const int last = min(end, n);

  const Rows x1 = rows_of<T>(a.x1, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n, 0, a.d1);
  const Rows x2 = rows_of<T>(a.x2, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n, 0, a.d1);
  const Rows x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
  const Rows y = rows_of<T>(a.y, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
  Tile<T, C, D1, NTH, VEC> p1, p2;
  Tile<T, C, D2, NTH, VEC> p3;
  p1.load(x1, begin, min(C, last - begin), tid);
  p2.load(x2, begin, min(C, last - begin), tid);
  p3.load(x3, begin, min(C, last - begin), tid);

  // the state: rows 16 kt + 4 g ... + 3 of the wave's half, column col0 + 16 part + lane % 16
  f32x4 U[KT];
  const long long uat = (A.nseg > 1 ? (long long)bh * A.nseg + seg : bh) * a.d1 * a.d2;
  const int uc = col0 + 16 * part + (lane & 15), ur = half * (D1 / H);
  if (a.u_in != nullptr) {
    load_state<KT, VEC>(U, a.u_in + uat, a.d1, a.d2, a.transposed, uc, lane >> 4, ur);
  } else {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) U[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // Tiles of P above the diagonal that a product over 32 keys reads: zero from here on, never written again.
  for (int e = tid; e < C * RBP / 16; e += NTH) lds_put(tp + 16 * e, u32x4{0, 0, 0, 0});
  put_weights<C>(tw, a2, C, a.off, a.su, tid);
  if (tid < C + 15) lds_put(td + 4 * tid, a.sp * power(a2, max(tid - 15, 0)));
  if (tid < C) lds_put(tl + 4 * tid, a.sr * power(a2, tid + 1 - a.off));
  const float gC = power(a2, C);

  f32x4 out[QT];
  // rows 16 qt + lane % 16 of the chunk at r0
  const auto put_rows = [&](int r0, int nr, Lane l, int qt0, int step) {
    const Buffer yb = y.rows(r0, nr);
    const unsigned c = (unsigned)((16 * part + 4 * l.g) * (int)sizeof(T)), row = y.offset(l.i, nr);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      if (qt % step != qt0) continue;
      if (VEC) {
        O::store4(yb, c < y.width ? row + (unsigned)y.step(16 * qt) + c : kNowhere, out[qt]);
      } else if (16 * qt + l.i < nr && c < y.width) {
        O::store_loose(y.at(r0 + 16 * qt + l.i) + c, (int)(y.width - c), out[qt]);
      }
    }
  };
  // Halves: each stores every second row tile, with what the other half has left of it in LDS.
  const auto join_rows = [&](int r0, int nr) {
    const Lane l = fresh<D1>(lane);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
      if (qt % 2 == half) out[qt] += lds_get<f32x4>(te + (part * QT + qt) * 1024 + 16 * (16 * l.g + l.i));
    if (a.y != nullptr) put_rows(r0, nr, l, half, 2);
  };

  for (int r0 = begin; r0 < last; r0 += C) {
    const int nr = min(C, last - r0);
    lds_barrier();   // the tiles' readers are done
    if (H == 2 && r0 > begin) join_rows(r0 - C, C);
    p1.store(t1, tid);
    p2.store(t2, tid);
    p3.store(t3, tid);
    if (nr < C) put_weights<C>(tw, a2, nr, a.off, a.su, tid);
    lds_barrier();
    if (r0 + C < last) {
      const int next = min(C, last - r0 - C);
      p1.load(x1, r0 + C, next, tid);
      p2.load(x2, r0 + C, next, tid);
      p3.load(x3, r0 + C, next, tid);
    }
    // P: the tiles on and below the diagonal, dealt out to the waves
    const Lane l = fresh<D1>(lane);
    const int b1 = O::template row_base<RB1>(l);
#pragma unroll
    for (int i = 0; i < (QT * (QT + 1) / 2 + W - 1) / W; ++i) {
      const int t = wave + W * i;
      if (t < QT * (QT + 1) / 2) {
        const int qt = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, kt = t - qt * (qt + 1) / 2;
        f32x4 s;
#pragma unroll
        for (int k = 0; k < K1; ++k) s = O::mma(O::row(t2 + kt * 16 * RB1, b1, k), O::row(t1 + qt * 16 * RB1, b1, k), k > 0 ? s : f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] *= lds_get<float>(td + 64 * (qt - kt) + 4 * (3 - j) + 4 * (l.i - 4 * l.g + 12));
        if (qt == kt) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[j] = l.i - 4 * l.g - j >= 0 ? s[j] : 0.f;
        }
        O::put4(tp + qt * 16 * RBP, O::template put_base<RBP>(l), kt, s);
        hold();
      }
    }
    const int bu = b1 ^ (half * (RB1 / H));
#pragma unroll
    for (int k = 0; k < K1 / H; ++k) {
      const typename O::frag u = O::state(U[2 * k], U[2 * k + 1]);
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
        out[qt] = O::mma(u, O::row(t1 + qt * 16 * RB1, bu, k), k > 0 ? out[qt] : f32x4{0.f, 0.f, 0.f, 0.f});
      hold();
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) out[qt] *= lds_get<float>(tl + 64 * qt + 4 * l.i);
    lds_barrier();   // P is there
    {
      const int b3 = O::template col_base<RB2>(l), bp = O::template row_base<RBP>(l);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (H == 2 && half != ks) continue;
        const typename O::frag v = O::template col<RB2>(t3 + 32 * ks * RB2, b3, part);
#pragma unroll
        for (int qt = 2 * ks; qt < QT; ++qt) out[qt] = O::mma(v, O::row(tp + qt * 16 * RBP, bp, ks), out[qt]);
        hold();
      }
    }
    if (H == 2) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
        if (qt % 2 != half) lds_put(te + (part * QT + qt) * 1024 + 16 * (16 * l.g + l.i), out[qt]);
    } else if (a.y != nullptr) {
      put_rows(r0, nr, l, 0, 1);
    }
    if (r0 + C < last || (last == n && a.u_out != nullptr)) {
      const float gn = nr < C ? power(a2, nr) : gC;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) U[kt] *= gn;
      update<T, C, D1, D2, H>(U, t2, t3, tw, 1.f, part, l, half);
    }
  }
  if (H == 2 && last > begin) {
    lds_barrier();
    const int r0 = begin + (last - begin - 1) / C * C;
    join_rows(r0, last - r0);
  }
  if (last == n && a.u_out != nullptr) store_state<KT>(U, a.u_out + (long long)bh * a.d1 * a.d2, a.d1, a.d2, uc, lane >> 4, ur);
}

template <typename T, int D1, int D2, bool VEC>
__global__ __launch_bounds__(4 * D2 * halves(D1), state_waves(D1)) void k_decay_state(States A) {
  typedef Op<T> O;
  constexpr int H = halves(D1), C = O::kChunk, KT = D1 / 16 / H, NTH = 4 * D2 * H;
  constexpr int t2 = 0, t3 = t2 + C * D1 * (int)sizeof(T), tw = t3 + C * D2 * (int)sizeof(T);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int part = wave % (D2 / 16), half = H == 2 ? wave / (D2 / 16) : 0;
  State a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  const int segs = A.nseg - 1, bh = blockIdx.x / segs, seg = blockIdx.x % segs, b = bh / A.H, h = bh % A.H, col0 = blockIdx.y * D2;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const int begin = seg * A.seg_len, end = begin + A.seg_len, cols = min(a.d2 - col0, D2);
  if (end >= n) return;   // nothing follows
  const float a2 = decay_log2(A.log_decay, h);
  const Rows x2 = rows_of<T>(a.x2, b, h, A.H, A.L, a.d1, A.layout, a.reverse, n, 0, a.d1);
  const Rows x3 = rows_of<T>(a.x3, b, h, A.H, A.L, a.d2, A.layout, a.reverse, n, col0, cols);
  Tile<T, C, D1, NTH, VEC> p2;
  Tile<T, C, D2, NTH, VEC> p3;
  // From the segment's end to its beginning, where the scan starts: what was read last is still in the memory-side cache then.
  p2.load(x2, end - C, C, tid);
  p3.load(x3, end - C, C, tid);
  f32x4 U[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) U[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  put_weights<C>(tw, a2, C, a.off, a.su, tid);
  for (int r0 = end - C; r0 >= begin; r0 -= C) {
    lds_barrier();
    p2.store(t2, tid);
    p3.store(t3, tid);
    lds_barrier();
    if (r0 > begin) {
      p2.load(x2, r0 - C, C, tid);
      p3.load(x3, r0 - C, C, tid);
    }
    update<T, C, D1, D2, H>(U, t2, t3, tw, power(a2, end - C - r0), part, fresh<D1>(lane), half);
  }
  store_state<KT>(U, a.seg + ((long long)bh * A.nseg + seg) * a.d1 * a.d2, a.d1, a.d2, col0 + 16 * part + (lane & 15), lane >> 4, half * (D1 / H));
}

template <typename T, int D1, int D2, bool VEC>
static dark_status launch(const Scans& a, int n, hipStream_t st) {
  constexpr int lds = scan_lds<T, D1, D2>();
  DARK_TRY(allow_lds(k_decay_scan<T, D1, D2, VEC>, lds));
  int d1, d2;
  widths_of(a, n, &d1, &d2);
  const dim3 grid((unsigned)((long long)a.B * a.H * a.nseg), (unsigned)((d2 + D2 - 1) / D2), (unsigned)n);
  DARK_LAUNCH(KID_DECAY_SCAN, st, (k_decay_scan<T, D1, D2, VEC>), grid, dim3(4 * D2 * halves(D1)), lds, a);
  return DARK_OK;
}
template <typename T, int D1, int D2, bool VEC>
static dark_status launch(const States& a, int n, hipStream_t st) {
  constexpr int lds = state_lds<T, D1, D2>();
  DARK_TRY(allow_lds(k_decay_state<T, D1, D2, VEC>, lds));
  const dim3 grid((unsigned)((long long)a.B * a.H * (a.nseg - 1)), (unsigned)((a.s[0].d2 + D2 - 1) / D2), (unsigned)n);
  DARK_LAUNCH(KID_DECAY_STATE, st, (k_decay_state<T, D1, D2, VEC>), grid, dim3(4 * D2 * halves(D1)), lds, a);
  return DARK_OK;
}

// The instance that holds d1 inner values, with 64 columns a workgroup where x3 has no more (or the state of 256 x 128 would take
// half of the registers) or the plan wants them, else 128.
template <typename T, int D1, int D2, typename A>
static dark_status pick(const A& a, int n, hipStream_t st) {
  const bool vec = a.s[0].d1 * sizeof(T) % 16 == 0 && a.s[0].d2 * sizeof(T) % 16 == 0;   // the same two in every scan
  return vec ? launch<T, D1, D2, true>(a, n, st) : launch<T, D1, D2, false>(a, n, st);
}
template <typename T, typename A>
static dark_status pick(const A& a, int n, hipStream_t st) {
  int d1, d2;
  widths_of(a, n, &d1, &d2);
  if (a.narrow) d2 = 64;
  if (d1 > 128) return pick<T, 256, 64>(a, n, st);
  if (d1 > 64) return d2 <= 64 ? pick<T, 128, 64>(a, n, st) : pick<T, 128, 128>(a, n, st);
  return d2 <= 64 ? pick<T, 64, 64>(a, n, st) : pick<T, 64, 128>(a, n, st);
}

}  // namespace decay
}  // namespace dark
