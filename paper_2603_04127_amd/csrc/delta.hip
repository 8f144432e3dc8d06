// The gated delta rule: argument checks, the launches of a call and the one-token recurrence.  The chunked kernels are in delta_scan.h, delta_team.h
// and delta_grad.h.
#include <algorithm>
#include <cmath>

#include "delta.h"

namespace dark {
namespace delta {
namespace {

constexpr int kMostWidth = 256;
constexpr long long kMostRows = 1LL << 28;
constexpr long long kMostHeads = 1 << 22;        // 768 threads each at most
constexpr long long kMostThreads = 1LL << 32;    // of a launch in one dimension, less one

// ---------------------------------------------------------------------------
// One token.  With D = a S: u = beta (v - D^T k), S' = D + k u^T, out = scale (D^T q + (q . k) u): one reduction over the rows for both
// readouts, and the state read and written once.  256 threads as `tx` units of W columns by 256 / tx rows; a thread holds its rows of
// the state (16 at most) in registers.  Bound by memory: 2048 states of 128 x 128, four beams a parent, 52 us, 5.2 TB/s; 16 of them 5 us, a launch.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float ld(const T* p);
template <>
__device__ __forceinline__ float ld<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ld<unsigned short>(const unsigned short* p) { return __uint_as_float((unsigned)*p << 16); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(unsigned short* p, float v) { *p = (unsigned short)fz::pack_bf16(v, 0.f); }

constexpr int kHeld = 16;

template <typename T, int W>
__global__ __launch_bounds__(256) void k_delta_step(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
                                                    const float* __restrict__ log_gate, const float* __restrict__ beta,
                                                    const int32_t* __restrict__ parent, int state_rows, const float* S_in, float* S_out,
                                                    T* __restrict__ out, int H, int dk, int dv, int tx, float scale) {
  typedef float vec __attribute__((ext_vector_type(W)));
  __shared__ float qs[kMostWidth], ks[kMostWidth];
  __shared__ vec part[2][256];
  __shared__ float dots[4];
  const int tid = threadIdx.x, b = blockIdx.x / H, h = blockIdx.x % H, x = tid % tx, row0 = tid / tx, rows = 256 / tx;
  const int c = (blockIdx.y * tx + x) * W;
  const bool mine = c < dv;
  const int from = parent != nullptr ? parent[b] : b;
  const bool there = (unsigned)from < (unsigned)state_rows;   // no such row: an empty state
  const long long size = (long long)dk * dv;
  const float* const Si = S_in + ((long long)(there ? from : 0) * H + h) * size + c;
  float* const So = S_out + (long long)blockIdx.x * size + c;
  vec s[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int i = row0 + u * rows;
    s[u] = 0.f;
    if (mine && there && i < dk) s[u] = *reinterpret_cast<const vec*>(Si + (long long)i * dv);
  }
  const float gate = log_gate != nullptr ? expf(log_gate[blockIdx.x]) : 1.f, be = beta[blockIdx.x];
  vec vv = 0.f;
  if (mine) {
#pragma unroll
    for (int j = 0; j < W; ++j) vv[j] = ld<T>(v + (long long)blockIdx.x * dv + c + j);
  }
  float qk = 0.f;
  if (tid < dk) {
    qs[tid] = ld<T>(q + (long long)blockIdx.x * dk + tid);
    ks[tid] = ld<T>(k + (long long)blockIdx.x * dk + tid);
    qk = qs[tid] * ks[tid];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) qk += __shfl_xor(qk, o, 64);
  if ((tid & 63) == 0) dots[tid >> 6] = qk;
  __syncthreads();
  qk = (dots[0] + dots[1]) + (dots[2] + dots[3]);
  vec ak = 0.f, aq = 0.f;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int i = row0 + u * rows;
    if (i < dk) {
      s[u] *= gate;
      ak += ks[i] * s[u];
      aq += qs[i] * s[u];
    }
  }
  part[0][tid] = ak;
  part[1][tid] = aq;
  __syncthreads();
  for (int o = 128; o >= tx; o >>= 1) {   // tx is a power of two
    if (tid < o) {
      part[0][tid] += part[0][tid + o];
      part[1][tid] += part[1][tid + o];
    }
    __syncthreads();
  }
  const vec u = be * (vv - part[0][x]);
  if (mine) {
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
      const int i = row0 + e * rows;
      if (i < dk) *reinterpret_cast<vec*>(So + (long long)i * dv) = s[e] + ks[i] * u;
    }
    if (row0 == 0) {
      const vec o = scale * (part[1][x] + qk * u);
#pragma unroll
      for (int j = 0; j < W; ++j) st(out + (long long)blockIdx.x * dv + c + j, o[j]);
    }
  }
}

}  // namespace

static dark_status check_params(const dark_delta_params* p, Problem* out) {
  if (p == nullptr) return DARK_EINVAL;
  if (p->B < 0 || p->L < 0 || p->H <= 0 || p->dk <= 0 || p->dv <= 0) return DARK_EINVAL;
  if (p->io_dtype != DARK_F32 && p->io_dtype != DARK_BF16) return DARK_EINVAL;
  if (p->layout != DARK_BHLD && p->layout != DARK_BLHD) return DARK_EINVAL;
  if (!(p->scale >= 0.f) || std::isinf(p->scale)) return DARK_EINVAL;
  const long long heads = (long long)p->B * p->H;
  if (p->dk > kMostWidth || p->dv > kMostWidth || heads > kMostHeads || (heads > 0 && p->L > kMostRows / heads)) return DARK_EUNSUPPORTED;
  // a chunk's rows are addressed by 32-bit offsets: 64 rows of all heads stay under 2^31 bytes
  if (p->layout == DARK_BLHD && (long long)p->H * (p->dk > p->dv ? p->dk : p->dv) > (1 << 22)) return DARK_EUNSUPPORTED;
  out->p = *p;
  out->scale = p->scale > 0.f ? p->scale : 1.0f / std::sqrt((float)p->dk);
  out->st = nullptr;
  return DARK_OK;
}

// A chunk's triangles take 256 threads: 2^28 rows make 12.4 million chunks at most, of sequences of 65 rows in fp32.  Its gradients (k_delta_grad) take 512
// where keys are wider than 64.
static bool too_many_chunks(const Problem& pb) {
  const int C = chunk_of(pb.p.io_dtype);
  return pb.BH() * ((pb.p.L + C - 1) / C) * (inner_of(pb.p.dk) > 64 ? 512 : 256) >= kMostThreads;
}

static Args args_of(const Problem& pb) {
  Args a = {};
  const int C = chunk_of(pb.p.io_dtype);
  a.B = pb.p.B;
  a.H = pb.p.H;
  a.L = pb.p.L;
  a.dk = pb.p.dk;
  a.dv = pb.p.dv;
  a.layout = pb.p.layout;
  a.chunks = (pb.p.L + C - 1) / C;
  a.dvp = (pb.p.dv + 63) / 64 * 64;
  a.scale = pb.scale;
  return a;
}

// The scratch of a call.
static void plan(const Problem& pb, Arena& ar, bool backward, Args* a) {
  const int C = chunk_of(pb.p.io_dtype), NB = blocks_of(C);
  const size_t chunks = (size_t)pb.BH() * a->chunks, inner = inner_of(pb.p.dk);
  a->tri = ar.take<fz::u32x4>(chunks * NB * 192);
  a->pri = ar.take<fz::u32x4>(chunks * NB * (pb.p.io_dtype == DARK_BF16 && !backward ? 128 : 192));
  a->vec = ar.take<float>(chunks * kVecs * C);
  if (!backward) return;
  a->trit = ar.take<fz::u32x4>(chunks * NB * 192);
  a->states = ar.take<float>(chunks * inner * a->dvp);
  a->dstates = ar.take<float>(chunks * inner * a->dvp);
  a->u = ar.take<float>(chunks * C * a->dvp);
  a->dr = ar.take<float>(chunks * C * a->dvp);
}

static dark_status prep(const Problem& pb, const Args& a, bool backward) {
  return pb.p.io_dtype == DARK_BF16 ? launch_prep_bf16(a, backward, pb.st) : launch_prep_f32(a, backward, pb.st);
}
static dark_status scan(const Problem& pb, const Args& a) {
  if (pb.p.io_dtype == DARK_BF16) return team_bf16(a) ? launch_team_bf16(a, pb.st) : launch_scan_bf16(a, pb.st);
  return team_f32(a) ? launch_team_f32(a, pb.st) : launch_scan_f32(a, pb.st);
}
static dark_status back(const Problem& pb, const Args& a, const float* g_in, float* g_out, bool states) {
  if (pb.p.io_dtype == DARK_BF16)
    return team_back_bf16(a, states) ? launch_team_back_bf16(a, g_in, g_out, states, pb.st) : launch_back_bf16(a, g_in, g_out, states, pb.st);
  return team_back_f32(a, states) ? launch_team_back_f32(a, g_in, g_out, states, pb.st) : launch_back_f32(a, g_in, g_out, states, pb.st);
}

static dark_status step(const Problem& pb, const void* q, const void* k, const void* v, const float* log_gate, const float* beta,
                        const int32_t* parent, int state_rows, const float* S_in, float* S_out, void* out) {
  const int dk = pb.p.dk, dv = pb.p.dv, H = pb.p.H;
  const int W = dv % 4 == 0 ? 4 : 1, units = (dv + W - 1) / W;
  // Columns of a workgroup: as many as leave a thread 16 rows at most, or fewer (16 at least, 64 bytes of a row) until there are four
  // workgroups a CU.
  int tx = 1;
  while (tx < units && (long long)2 * tx * dk <= 256 * kHeld) tx *= 2;
  const int least = 16 / W;
  while (tx > least && pb.BH() * ((units + tx - 1) / tx) < 1024) tx /= 2;
  const dim3 grid((unsigned)pb.BH(), (unsigned)((units + tx - 1) / tx));
#define DARK_STEP(T, WW)                                                                                                        \
  DARK_LAUNCH(KID_DELTA_STEP, pb.st, (k_delta_step<T, WW>), grid, dim3(256), 0, static_cast<const T*>(q), static_cast<const T*>(k), \
              static_cast<const T*>(v), log_gate, beta, parent, state_rows, S_in, S_out, static_cast<T*>(out), H, dk, dv, tx, pb.scale)
  if (pb.p.io_dtype == DARK_BF16) {
    if (W == 4) DARK_STEP(unsigned short, 4);
    else DARK_STEP(unsigned short, 1);
  } else {
    if (W == 4) DARK_STEP(float, 4);
    else DARK_STEP(float, 1);
  }
#undef DARK_STEP
  return DARK_OK;
}

}  // namespace delta
}  // namespace dark

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------
using namespace dark;

namespace {
size_t size_of(const dark_delta_params& p) { return p.io_dtype == DARK_BF16 ? 2 : 4; }
// Bytes of Q or K, of V, of the gates, of a state.
struct Sizes {
  size_t k, v, gate, state, lengths;
  explicit Sizes(const delta::Problem& pb) {
    const size_t rows = (size_t)pb.BH() * pb.p.L;
    k = rows * pb.p.dk * size_of(pb.p);
    v = rows * pb.p.dv * size_of(pb.p);
    gate = rows * sizeof(float);
    state = (size_t)pb.BH() * pb.p.dk * pb.p.dv * sizeof(float);
    lengths = (size_t)pb.p.B * sizeof(int32_t);
  }
};
size_t measure(const delta::Problem& pb, bool backward) {
  if (pb.p.B == 0 || pb.p.L == 0) return 0;
  Arena ar(nullptr, 0);
  delta::Args a = delta::args_of(pb);
  delta::plan(pb, ar, backward, &a);
  return ar.off;
}
dark_status check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return DARK_OK;
  if (ws == nullptr || ws_bytes < need) return DARK_EWORKSPACE;
  return aligned(ws, 256) ? DARK_OK : DARK_EALIGN;
}
}  // namespace

extern "C" {

size_t dark_delta_workspace_bytes(const dark_delta_params* p, int backward) {
  delta::Problem pb;
  if (delta::check_params(p, &pb) != DARK_OK || (backward != 0 && delta::too_many_chunks(pb))) return 0;
  return measure(pb, backward != 0);
}

dark_status dark_delta_fwd(const dark_delta_params* p, const void* Q, const void* K, const void* V, const float* log_gate,
                           const float* beta, const int32_t* lengths, const float* S_in, void* out, float* S_out, void* ws,
                           size_t ws_bytes, void* hip_stream) {
  delta::Problem pb;
  DARK_TRY(delta::check_params(p, &pb));
  if (pb.p.B == 0 || (pb.p.L == 0 && S_out == nullptr)) return DARK_OK;
  if (pb.p.L > 0 && (!Q || !K || !V || !beta || !out)) return DARK_EINVAL;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(S_in, 16) || !aligned(S_out, 16) ||
      !aligned(log_gate, 4) || !aligned(beta, 4) || !aligned(lengths, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  if (S_in != S_out && overlap({S_in, n.state}, {S_out, n.state})) return DARK_EINVAL;
  DARK_TRY(check_workspace(ws, ws_bytes, measure(pb, false)));
  if (overlap({{out, n.v}, {S_out, n.state}}, {{Q, n.k}, {K, n.k}, {V, n.v}, {log_gate, n.gate}, {beta, n.gate}, {lengths, n.lengths}}) ||
      overlap({out, n.v}, {S_in, n.state}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  Arena ar(ws, ws_bytes);
  delta::Args a = delta::args_of(pb);
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.log_gate = log_gate;
  a.beta = beta;
  a.lengths = lengths;
  a.out = out;
  a.s_in = S_in;
  a.s_out = S_out;
  if (pb.p.L > 0) {
    delta::plan(pb, ar, false, &a);
    if (ar.overflow) return DARK_EWORKSPACE;
    DARK_TRY(delta::prep(pb, a, false));
  }
  return delta::scan(pb, a);
}

dark_status dark_delta_bwd(const dark_delta_params* p, const void* Q, const void* K, const void* V, const float* log_gate,
                           const float* beta, const int32_t* lengths, const float* S_in, const void* dOut, const float* dS_out, void* dQ,
                           void* dK, void* dV, float* dlog_gate, float* dbeta, float* dS_in, void* ws, size_t ws_bytes, void* hip_stream) {
  delta::Problem pb;
  DARK_TRY(delta::check_params(p, &pb));
  if (delta::too_many_chunks(pb)) return DARK_EUNSUPPORTED;
  if (pb.p.B == 0 || (pb.p.L == 0 && dS_in == nullptr)) return DARK_OK;
  if (pb.p.L > 0 && (!Q || !K || !V || !beta || !dOut)) return DARK_EINVAL;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(dOut, 16) || !aligned(S_in, 16) || !aligned(dS_out, 16) ||
      !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16) || !aligned(dS_in, 16) || !aligned(log_gate, 4) || !aligned(beta, 4) ||
      !aligned(dlog_gate, 4) || !aligned(dbeta, 4) || !aligned(lengths, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  DARK_TRY(check_workspace(ws, ws_bytes, measure(pb, true)));
  if (overlap({{dQ, n.k}, {dK, n.k}, {dV, n.v}, {dlog_gate, n.gate}, {dbeta, n.gate}, {dS_in, n.state}},
              {{Q, n.k}, {K, n.k}, {V, n.v}, {dOut, n.v}, {log_gate, n.gate}, {beta, n.gate}, {S_in, n.state}, {dS_out, n.state}, {lengths, n.lengths}}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  Arena ar(ws, ws_bytes);
  delta::Args a = delta::args_of(pb);
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.log_gate = log_gate;
  a.beta = beta;
  a.lengths = lengths;
  a.dOut = dOut;
  a.dQ = dQ;
  a.dK = dK;
  a.dV = dV;
  a.dgate = dlog_gate;
  a.dbeta = dbeta;
  const bool grads = dQ != nullptr || dK != nullptr || dV != nullptr || dlog_gate != nullptr || dbeta != nullptr;
  if (!grads && dS_in == nullptr) return DARK_OK;
  if (pb.p.L > 0) {
    delta::plan(pb, ar, true, &a);
    if (ar.overflow) return DARK_EWORKSPACE;
    DARK_TRY(delta::prep(pb, a, true));
  }
  a.s_in = S_in;
  DARK_TRY(delta::back(pb, a, dS_out, dS_in, grads && pb.p.L > 0));
  if (!grads || pb.p.L == 0) return DARK_OK;
  return pb.p.io_dtype == DARK_BF16 ? delta::launch_grad_bf16(a, pb.st) : delta::launch_grad_f32(a, pb.st);
}

dark_status dark_delta_step(const dark_delta_params* p, const void* q, const void* k, const void* v, const float* log_gate,
                            const float* beta, const int32_t* parent, int state_rows, const float* S_in, float* S_out, void* out,
                            void* hip_stream) {
  delta::Problem pb;
  if (p == nullptr) return DARK_EINVAL;
  dark_delta_params one = *p;
  one.L = 1;
  DARK_TRY(delta::check_params(&one, &pb));
  if (pb.p.B == 0) return DARK_OK;
  if (!q || !k || !v || !beta || !S_in || !S_out || !out) return DARK_EINVAL;
  if (parent == nullptr ? state_rows != pb.p.B : state_rows <= 0) return DARK_EINVAL;
  const size_t elem = size_of(pb.p);   // rows of one tensor, slices of a longer one: no more is asked of them
  if (!aligned(q, elem) || !aligned(k, elem) || !aligned(v, elem) || !aligned(out, elem) || !aligned(S_in, 16) || !aligned(S_out, 16) ||
      !aligned(log_gate, 4) || !aligned(beta, 4) || !aligned(parent, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  const size_t past = n.state / pb.p.B * state_rows;
  if ((parent != nullptr || S_in != S_out) && overlap({S_in, past}, {S_out, n.state})) return DARK_EINVAL;
  if (overlap({{out, n.v}, {S_out, n.state}}, {{q, n.k}, {k, n.k}, {v, n.v}, {log_gate, n.gate}, {beta, n.gate}, {parent, n.lengths}}) ||
      overlap({out, n.v}, {S_in, past}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  return delta::step(pb, q, k, v, log_gate, beta, parent, state_rows, S_in, S_out, out);
}

}  // extern "C"
