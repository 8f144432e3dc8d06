// The gated delta rule: what its translation units share.
//
// Per (b,h), with a_t = exp(log_gate_t), from a state S_0 [dk, dv]:
//   u_t = beta_t (v_t - a_t S_(t-1)^T k_t),   S_t = a_t S_(t-1) + k_t u_t^T,   o_t = scale S_t^T q_t.
// A chunk of C rows from the state S before it, with G_t the sum of the chunk's log gates up to row t, gamma_t = exp(G_t),
// left_t = exp(G_C - G_t), Gamma = exp(G_C), D_ti = exp(G_t - G_i) for i <= t, E_ti = D_ti (k_t . k_i) for i < t (zero elsewhere):
//   T = (I + diag(beta) E)^-1,   P = D o (Q K^T),
//   R = diag(beta) (V - diag(gamma) K S),   U = T R,   O = scale (diag(gamma) Q S + P U),   S' = Gamma S + K^T diag(left) U.
// Every exponent that is formed is a sum of gates of consecutive tokens: with gates <= 0 nothing overflows.
// Backward, from the gradient G' of the state behind the chunk (below: dS'):
//   dU = scale P^T dO + diag(left) K dS',   dR = T^T dU,   dV = diag(beta) dR,
//   dS = Gamma dS' + scale Q^T diag(gamma) dO - K^T diag(gamma beta) dR,
//   N = scale D o (dO U^T),   M = -diag(beta) (D o (dR U^T)) below the diagonal,
//   dQ = scale diag(gamma) dO S^T + N K,
//   dK = -diag(gamma beta) dR S^T + diag(left) U dS'^T + M K + M^T K + N^T Q,
//   dbeta_t = dR_t . v_t - gamma_t k_t . (S dR_t) - sum_(i<t) E_ti (dR_t . u_i),
// and the gradient of log gate t sums, over all weights exp(G_r - G_i) with i < t <= r, the weight times its gradient.
// Two kernels forward: k_delta_prep (T and P of every chunk, in parallel) and k_delta_scan (chunk after chunk); three backward: k_delta_prep,
// k_delta_back (the states and U, chunk after chunk, and, beside them, dS' and dR, from the last chunk to the first: neither asks for the other) and
// k_delta_grad (the rest, in parallel).  The scans have two forms: one wave for 16 columns of the state (delta_scan.h: any size), or a team of waves
// (delta_team.h: k_delta_team, k_delta_team_back).
#pragma once

#include "rows.h"

namespace dark {
namespace delta {

struct Problem {
  dark_delta_params p;
  float scale;    // resolved (never 0)
  hipStream_t st;
  long long BH() const { return (long long)p.B * p.H; }
};

// Rows of a chunk, blocks of 16 rows and 32 inner values that a lower triangle of C x C consists of as an operand.
constexpr int chunk_of(int io_dtype) { return io_dtype == DARK_BF16 ? 64 : 32; }
constexpr int blocks_of(int C) { return C == 64 ? 6 : 2; }
// Rows of C floats that k_delta_prep leaves for a chunk beside its operands: gamma, left, beta, Gamma (throughout), which the scans take, and G as
// the sum of two floats.
constexpr int kVecs = 6, kScanVecs = 4;

struct Args {
  const void *Q, *K, *V, *dOut;
  const float *log_gate, *beta;
  const int32_t* lengths;
  void *out, *dQ, *dK, *dV;
  float *dgate, *dbeta;
  const float* s_in;      // state before the first row; null: zero
  float* s_out;           // state behind the last row; null: not asked for
  int B, H, L, dk, dv, layout, chunks;
  int dvp;                // columns of scratch states and rows: dv, rounded up to 64
  float scale;
  // scratch, for every (b,h) and chunk
  fz::u32x4* tri;         // T in operand order: 3 planes of blocks_of(C) x 64 lanes x 8 values
  fz::u32x4* trit;        // T^T (backward)
  fz::u32x4* pri;         // P, as many planes as an output takes; backward: P^T scale, 3 planes
  float* vec;             // kVecs x C floats
  float* states;          // [D1, dvp], before the chunk
  float* dstates;         // [D1, dvp], gradient of the state behind the chunk
  float *u, *dr;          // [C, dvp]
};

dark_status launch_prep_bf16(const Args& a, bool backward, hipStream_t st);
dark_status launch_prep_f32(const Args& a, bool backward, hipStream_t st);
dark_status launch_scan_bf16(const Args& a, hipStream_t st);
dark_status launch_scan_f32(const Args& a, hipStream_t st);
// Backward, in one launch: from the last chunk to the first from the gradient g_in of the state behind it to g_out, of that before the first; and, if asked
// for, the states before the chunks, and U.
dark_status launch_back_bf16(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st);
dark_status launch_back_f32(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st);
dark_status launch_grad_bf16(const Args& a, hipStream_t st);
dark_status launch_grad_f32(const Args& a, hipStream_t st);

// A team of waves for 16 columns (delta_team.h), and whether a call takes it.
bool team_bf16(const Args& a);
bool team_f32(const Args& a);
bool team_back_bf16(const Args& a, bool states);
bool team_back_f32(const Args& a, bool states);
dark_status launch_team_bf16(const Args& a, hipStream_t st);
dark_status launch_team_f32(const Args& a, hipStream_t st);
dark_status launch_team_back_bf16(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st);
dark_status launch_team_back_f32(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st);

// Rows of the state that the kernels hold.
inline int inner_of(int dk) { return dk > 128 ? 256 : dk > 64 ? 128 : 64; }

}  // namespace delta
}  // namespace dark
