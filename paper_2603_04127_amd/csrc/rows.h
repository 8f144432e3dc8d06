// Rows of sequences and tiles of states on their way between memory, LDS and registers: what the chunked kernels of linear attention
// (decayed, gated delta rule) share.
#pragma once

#include "fused_common.h"

namespace dark {
namespace rows {

using namespace fz;

// A lane of a wave whose products take 16 rows or columns in four groups of lanes.
struct Lane {
  int i, g;   // lane % 16, lane / 16
};

// LDS by its address.  These kernels have dynamic LDS alone, which begins at 0; by way of a pointer to it the compiler adds that
// 0 to every address, a sixth of the scan's vector instructions.
template <typename V>
using Lds = __attribute__((address_space(3))) V;
template <typename V>
__device__ static inline V lds_get(int at) { return *reinterpret_cast<const Lds<V>*>((unsigned)at); }
template <typename V>
__device__ static inline void lds_put(int at, V v) { *reinterpret_cast<Lds<V>*>((unsigned)at) = v; }
__device__ static inline u32x2 lds_get_tr16(int at) {
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<Lds<s16x4>*>((unsigned)at));
  return *reinterpret_cast<const u32x2*>(&v);
}

// Nothing is moved across: what one step has read is used up before the next step reads, so that 128 registers are enough.
__device__ static inline void hold() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Memory by buffer instructions: a wave-uniform address and extent, 32-bit offsets of the lanes.  What lies at or behind the extent
// reads as zero and is not written, so that rows behind a sequence, columns behind the last and parts of a tile need no branches:
// they are given offsets that are too large.
typedef __amdgpu_buffer_rsrc_t Buffer;
// (Extents of a chunk are wave-uniform; said so here, as the compiler loops over the lanes' values where it has computed one in a
// vector register.)
__device__ static inline Buffer buffer(const void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000);
}
constexpr unsigned kNowhere = 0x80000000u;   // every extent is smaller (the callers' checks)

// Rows of a (b,h), chunk by chunk.  Row r is token r, or counted from the end token n - 1 - r.
struct Rows {
  const char* head;   // token 0
  unsigned row;       // bytes from one token to the next
  unsigned width;     // bytes of a row that exist from the tile's first column on
  int n, reverse;
  // the tokens of rows r0 ... r0 + nr - 1
  __device__ Buffer rows(int r0, int nr) const {
    return buffer(head + (long long)(reverse ? n - r0 - nr : r0) * row, nr > 0 ? (unsigned)(nr - 1) * row + width : 0u);
  }
  // the same from a multiple of 4 bytes on, `skew` before the first of them, to a multiple of 4
  __device__ Buffer loose(int r0, int nr, unsigned& skew) const {
    const char* const p = head + (long long)(reverse ? n - r0 - nr : r0) * row;
    skew = (unsigned)reinterpret_cast<uintptr_t>(p) & 3u;
    return buffer(p - skew, nr > 0 ? ((unsigned)(nr - 1) * row + width + skew + 3u) & ~3u : 0u);
  }
  // row r of the sequence
  __device__ char* at(int r) const { return const_cast<char*>(head) + (long long)(reverse ? n - 1 - r : r) * row; }
  // offset of the chunk's row `row`, of nr; too large for a row that does not exist (negative, read as unsigned, where counted from the end)
  __device__ unsigned offset(int r, int nr) const { return (unsigned)(reverse ? nr - 1 - r : r) * row; }
  // from there to the row `by` rows further on
  __device__ int step(int by) const { return reverse ? -by * (int)row : by * (int)row; }
};
template <typename T>
__device__ static inline Rows rows_of(const void* x, int b, int h, int H, int L, int d, int layout, int reverse, int n, int col0, int cols) {
  const long long first = layout == DARK_BHLD ? ((long long)b * H + h) * L * d : ((long long)b * L * H + h) * d;
  return {static_cast<const char*>(x) + (first + col0) * (long long)sizeof(T), (unsigned)(layout == DARK_BHLD ? d : H * d) * (unsigned)sizeof(T),
          (unsigned)(cols * (int)sizeof(T)), n, reverse};
}

// 16 bytes of a row that begins anywhere, as they come: the whole words that hold them, and which of their bytes are the row's.
// (Element by element, every load waited for where it was issued: the training step of 24 heads of 1534, 33 and 65 wide, took 113 us.)
template <typename T>
struct Piece {
  u32x4 r;
  unsigned behind;   // 16-bit elements: what follows
  // at: where it begins in the buffer, or kNowhere
  __device__ void load(Buffer b, unsigned at) {
    r = __builtin_amdgcn_raw_buffer_load_b128(b, at & ~3u, 0, 0);
    if (sizeof(T) == 2) behind = __builtin_amdgcn_raw_buffer_load_b32(b, (at & ~3u) + 16u, 0, 0);
  }
  // the piece: `shift` is 16 where it begins in the middle of a word, `have` its bytes that exist
  __device__ u32x4 get(unsigned shift, int have) const {
    u32x4 v = r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (sizeof(T) == 2) v[j] = __builtin_amdgcn_alignbit(j < 3 ? r[j < 3 ? j + 1 : 3] : behind, r[j], shift);
      v[j] &= have >= 4 * j + 4 ? ~0u : have > 4 * j ? 0xffffu : 0u;
    }
    return v;
  }
};

// A wave's columns of a state [d1, d2] in memory (or of its transpose): rows r0 + 16 kt + 4 g ... + 3 of column c (behind the last: c >= d2).
template <int KT, bool VEC>
__device__ static inline void load_state(f32x4 (&U)[KT], const float* p, int d1, int d2, int transposed, int c, int g, int r0 = 0) {
  const Buffer b = buffer(p, (unsigned)(d1 * d2) * 4u);
  if (!transposed) {
    const unsigned off = c < d2 ? (unsigned)((r0 + 4 * g) * d2 + c) * 4u : kNowhere;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int j = 0; j < 4; ++j) U[kt][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off + (unsigned)((16 * kt + j) * d2) * 4u, 0, 0));
  } else {
    const unsigned off = c < d2 ? (unsigned)(c * d1 + r0 + 4 * g) * 4u : kNowhere;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const int row = r0 + 16 * kt + 4 * g;   // rows behind the last would be the next column
      if (VEC) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(b, row < d1 ? off + 64u * kt : kNowhere, 0, 0);
        __builtin_memcpy(&U[kt], &v, 16);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) U[kt][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, row + j < d1 ? off + 64u * kt + 4u * j : kNowhere, 0, 0));
      }
    }
  }
}
template <int KT>
__device__ static inline void store_state(const f32x4 (&U)[KT], float* p, int d1, int d2, int c, int g, int r0 = 0) {
  const Buffer b = buffer(p, (unsigned)(d1 * d2) * 4u);
  const unsigned off = c < d2 ? (unsigned)((r0 + 4 * g) * d2 + c) * 4u : kNowhere;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int j = 0; j < 4; ++j) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(U[kt][j]), b, off + (unsigned)((16 * kt + j) * d2) * 4u, 0, 0);
}

}  // namespace rows
}  // namespace dark
