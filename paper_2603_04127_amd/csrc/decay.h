// Linear attention with a decay for each head: what its translation units share.
//
// Forward, per (b,h) with g = exp(log_decay[h]):
//   S_t = g S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t.
// With G_t = g G_{t+1} + scale q_t dO_t^T (behind the last row: dS_n), the gradients are
//   dQ_t = scale S_t dO_t,  dK_t = G_t v_t,  dV_t = G_t^T k_t,  dS_0 = g G_1.
// So the forward pass and each of the three gradients are one and the same scan over rows r = 0, 1, ... of three operands, the
// latter two gradients with the rows counted from the sequence's end:
//   y_r = sp sum_{c <= r} g^(r-c) (x1_r . x2_c) x3_c + sr g^(r+1-off) U^T x1_r,   U the state before row 0,
//   state behind n rows: g^n U + su sum_c g^(n-1-c+off) x2_c x3_c^T.
//     out: x = (Q, K, V),  U = S_0,    sp = sr = scale, su = 1,  off = 0
//     dQ:  x = (dO, V, K), U = S_0^T,  sp = sr = scale, su = 1,  off = 0
//     dV:  x = (K, Q, dO), U = dS_n,   sp = su = scale, sr = 1,  off = 1, reversed   (state behind the rows: dS_0)
//     dK:  x = (V, dO, Q), U = dS_n^T, sp = su = scale, sr = 1,  off = 1, reversed
// Every power of g has an exponent >= 0: nothing overflows however strong the decay.
#pragma once

#include "fused_common.h"

namespace dark {
namespace decay {

struct Problem {
  dark_decay_params p;
  float scale;    // resolved (never 0)
  hipStream_t st;
  long long BH() const { return (long long)p.B * p.H; }
};

struct Scan {
  const void *x1, *x2, *x3;   // [B, H, L, d1], [B, H, L, d1], [B, H, L, d2], or with the heads behind the rows
  void* y;                    // like x3
  const float* u_in;          // state before row 0 of the sequence (one segment) or of every segment (several); null: zero
  float* u_out;               // state behind the last row; null: not asked for
  int d1, d2;
  int transposed;             // u_in is [.., d2, d1] instead of [.., d1, d2] (u_out never)
  int reverse, off;
  float sp, sr, su;
};
constexpr int kMostScans = 3;
struct Scans {
  Scan s[kMostScans];
  const float* log_decay;
  const int32_t* lengths;
  int B, H, L, layout;
  int nseg, seg_len;          // segments of a sequence; seg_len is a multiple of the chunk
  int narrow;                 // 64 columns a workgroup
};

// Segment states: su sum_c g^(len-1-c+off) x2_c x3_c^T over every segment that another one follows.
struct State {
  const void *x2, *x3;
  const float* u_in;          // state before row 0 of the sequence, null: zero
  float* seg;                 // [B, H, nseg, d1, d2]
  int d1, d2, reverse, off;
  float su;
};
struct States {
  State s[2];
  const float* log_decay;
  const int32_t* lengths;
  int B, H, L, layout, nseg, seg_len, narrow;
};

// Rows of a chunk: what the scan takes at a time.
constexpr int kChunkBf16 = 64, kChunkF32 = 32;

// The widths that hold all `n` scans (states).
template <typename A>
inline void widths_of(const A& a, int n, int* d1, int* d2) {
  *d1 = *d2 = 0;
  for (int i = 0; i < n; ++i) {
    *d1 = a.s[i].d1 > *d1 ? a.s[i].d1 : *d1;
    *d2 = a.s[i].d2 > *d2 ? a.s[i].d2 : *d2;
  }
}

dark_status launch_scan_bf16(const Scans& a, int n, hipStream_t st);
dark_status launch_scan_f32(const Scans& a, int n, hipStream_t st);
dark_status launch_state_bf16(const States& a, int n, hipStream_t st);
dark_status launch_state_f32(const States& a, int n, hipStream_t st);
// decay_short.hip: the same scans, one segment, without a state where nobody asks for it.
dark_status launch_short_bf16(const Scans& a, int n, hipStream_t st);

dark_status check_params(const dark_decay_params* p, Problem* out);
dark_status forward(const Problem& pb, Arena& ar, const void* Q, const void* K, const void* V, const float* log_decay,
                    const int32_t* lengths, const float* S_in, void* out, float* S_out);
dark_status backward(const Problem& pb, Arena& ar, const void* Q, const void* K, const void* V, const float* log_decay,
                     const int32_t* lengths, const float* S_in, const void* dOut, const float* dS_out, void* dQ, void* dK,
                     void* dV, float* dS_in);
dark_status step(const Problem& pb, const void* q, const void* k, const void* v, const float* log_decay,
                 const int32_t* parent, int state_rows, const float* S_in, float* S_out, void* out);

}  // namespace decay
}  // namespace dark
