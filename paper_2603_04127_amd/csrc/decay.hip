// Linear attention with a decay for each head: argument checks, the plan of a call, the prefix over segment states and the
// one-token recurrence.  The scan itself is in decay_scan.h.
#include <algorithm>
#include <cmath>

#include "decay.h"

namespace dark {
namespace decay {
namespace {

using fz::f32x4;
using fz::fast_exp2;
using fz::kLog2e;

// The states before every segment, in place of the segments' own: U_0 = u_in, U_(s+1) = g^len U_s + seg_s.  One thread an element
// (four where they divide), segment by segment, sixteen of them asked for at once; bound by reading and writing the states once (64 heads of
// 128 x 128, 8 segments: 63 MB in 12 to 14 us, the rate of a copy), few states by a launch and two trips to memory (4 us; 64 segments of one
// head 9).
template <int W>
__global__ __launch_bounds__(256) void k_decay_prefix(States A) {
  typedef float vec __attribute__((ext_vector_type(W)));
  State a = A.s[0];
  if (blockIdx.z == 1) a = A.s[1];
  const long long size = (long long)a.d1 * a.d2, e = ((long long)blockIdx.y * 256 + threadIdx.x) * W;
  if (e >= size) return;
  const int bh = blockIdx.x, b = bh / A.H, h = bh % A.H;
  const int n = A.lengths != nullptr ? min(max(A.lengths[b], 0), A.L) : A.L;
  const int used = max(1, (n + A.seg_len - 1) / A.seg_len);
  const float gl = fast_exp2(fmaxf(A.log_decay[h] * kLog2e, -1e30f) * (float)A.seg_len);
  vec U = 0.f;
  if (a.u_in != nullptr) U = *reinterpret_cast<const vec*>(a.u_in + bh * size + e);
  float* const s = a.seg + (long long)bh * A.nseg * size + e;
  constexpr int kAtOnce = 16;
  for (int i0 = 0; i0 < used - 1; i0 += kAtOnce) {
    vec own[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) own[i] = *reinterpret_cast<const vec*>(s + min(i0 + i, used - 2) * size);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (i0 + i < used - 1) {
        *reinterpret_cast<vec*>(s + (i0 + i) * size) = U;
        U = gl * U + own[i];
      }
    }
  }
  *reinterpret_cast<vec*>(s + (long long)(used - 1) * size) = U;
}

// A state that is updated in place while other workgroups still read it is read from a copy.
__global__ __launch_bounds__(256) void k_decay_copy(const float* __restrict__ from, float* __restrict__ to, long long n) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) to[i] = from[i];
}

// ---------------------------------------------------------------------------
// One token: S <- g S + k v^T, out = scale S^T q, for the columns of a workgroup.  Bound by reading and writing the state once
// (64 x 32 states of 128 x 128: 135 MB written and, as beams share parents, 93 read in 45 us, 5.1 TB/s; 16 states 4.6 us, a launch).
// 256 threads as `tx` units of W columns by 256 / tx rows; every thread sums its rows' share of the output, LDS joins the shares.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float ld(const T* p);
template <>
__device__ __forceinline__ float ld<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ld<unsigned short>(const unsigned short* p) { return __uint_as_float((unsigned)*p << 16); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(unsigned short* p, float v) { *p = (unsigned short)fz::pack_bf16(v, 0.f); }

constexpr int kMostWidth = 256;
constexpr long long kMostGroups = 1 << 22;   // along a grid's x: of 512 threads each they stay under the 2^32 that a launch can have
constexpr int kAhead = 8;   // rows in flight a thread

template <typename T, int W>
__global__ __launch_bounds__(256) void k_decay_step(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
                                                    const float* __restrict__ log_decay, const int32_t* __restrict__ parent, int state_rows,
                                                    const float* S_in, float* S_out, T* __restrict__ out, int H, int dk, int dv, int tx,
                                                    float scale) {
  typedef float vec __attribute__((ext_vector_type(W)));
  __shared__ float qs[kMostWidth], ks[kMostWidth];
  __shared__ vec part[256];
  const int tid = threadIdx.x, b = blockIdx.x / H, h = blockIdx.x % H, x = tid % tx, row0 = tid / tx, rows = 256 / tx;
  const int c = (blockIdx.y * tx + x) * W;
  const bool mine = c < dv;
  const int from = parent != nullptr ? parent[b] : b;
  const bool there = (unsigned)from < (unsigned)state_rows;   // no such row: an empty state
  const long long size = (long long)dk * dv;
  const float* const Si = S_in + ((long long)(there ? from : 0) * H + h) * size + c;
  float* const So = S_out + (long long)blockIdx.x * size + c;
  vec s[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int i = row0 + u * rows;
    s[u] = 0.f;
    if (mine && there && i < dk) s[u] = *reinterpret_cast<const vec*>(Si + (long long)i * dv);
  }
  const float gam = fast_exp2(fmaxf(log_decay[h] * kLog2e, -1e30f));
  vec vv = 0.f;
  if (mine) {
#pragma unroll
    for (int j = 0; j < W; ++j) vv[j] = ld<T>(v + (long long)blockIdx.x * dv + c + j);
  }
  if (tid < dk) {
    qs[tid] = scale * ld<T>(q + (long long)blockIdx.x * dk + tid);
    ks[tid] = ld<T>(k + (long long)blockIdx.x * dk + tid);
  }
  __syncthreads();
  vec acc = 0.f;
  for (int i0 = row0; i0 < dk; i0 += kAhead * rows) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u * rows;
      if (i < dk) {
        const vec n = gam * s[u] + ks[i] * vv;
        if (mine) *reinterpret_cast<vec*>(So + (long long)i * dv) = n;
        acc += qs[i] * n;
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + (kAhead + u) * rows;
      if (mine && there && i < dk) s[u] = *reinterpret_cast<const vec*>(Si + (long long)i * dv);
    }
  }
  part[tid] = acc;
  __syncthreads();
  for (int o = 128; o >= tx; o >>= 1) {   // tx is a power of two
    if (tid < o) part[tid] += part[tid + o];
    __syncthreads();
  }
  if (tid < tx && mine) {
#pragma unroll
    for (int j = 0; j < W; ++j) st(out + (long long)blockIdx.x * dv + c + j, part[tid][j]);
  }
}

}  // namespace

dark_status check_params(const dark_decay_params* p, Problem* out) {
  if (p == nullptr) return DARK_EINVAL;
  if (p->B < 0 || p->L < 0 || p->H <= 0 || p->dk <= 0 || p->dv <= 0) return DARK_EINVAL;
  if (p->io_dtype != DARK_F32 && p->io_dtype != DARK_BF16) return DARK_EINVAL;
  if (p->layout != DARK_BHLD && p->layout != DARK_BLHD) return DARK_EINVAL;
  if (!(p->scale >= 0.f) || std::isinf(p->scale) || p->sched_segments < 0) return DARK_EINVAL;
  if (p->dk > kMostWidth || p->dv > kMostWidth || (long long)p->B * p->H > kMostGroups || p->L > (1 << 30)) return DARK_EUNSUPPORTED;
  // a chunk's rows are addressed by 32-bit offsets: 64 rows of all heads stay under 2^31 bytes
  if (p->layout == DARK_BLHD && (long long)p->H * (p->dk > p->dv ? p->dk : p->dv) > (1 << 22)) return DARK_EUNSUPPORTED;
  out->p = *p;
  out->scale = p->scale > 0.f ? p->scale : 1.0f / std::sqrt((float)p->dk);
  out->st = nullptr;
  return DARK_OK;
}

namespace {

// How a call is laid out: one segment or several, or bf16 sequences of some chunks without states (decay_short.h).
struct Plan {
  int nseg = 1, seg_len = 0;
  bool narrow = false;   // 64 columns a workgroup
  bool direct = false;
};

// What the kernels take, in us, by the widths of their instances (d1, d2): a chunk of the scan while a CU has nothing else to do (the
// segment states take 0.45 of it), a step of the direct kernel, and how many (block, chunk) pairs a us that kernel gets through when
// the chip is full.  Measured on 8 heads of 1024 (fp32) and 2048 rows, and on 16 to 128 heads of 256 to 1024.
struct Cost {
  float bf16, f32, step, pairs;
};
Cost cost_of(int d1, int d2) {
  if (d1 > 128) return {3.9f, 7.2f, 2.9f, 120.f};
  if (d1 > 64) return d2 <= 64 ? Cost{2.6f, 4.5f, 1.8f, 250.f} : Cost{3.2f, 6.4f, 2.0f, 172.f};
  return d2 <= 64 ? Cost{1.9f, 2.8f, 1.4f, 335.f} : Cost{2.4f, 4.0f, 1.8f, 250.f};
}

// A launch costs 4 us and, on the CUs, its workgroups' chunks one after the other: workgroups beyond one a CU wait for it or share it,
// which comes to the same.  More segments shorten the chains until the chip is full; their states are written, and read and written
// once more by the prefix over them, and cost two launches.  Workgroups of 64 columns instead of 128 are another way to have more of
// them, with shorter chunks, each computing P for itself: fp32, bound by its products, gains while there are few chunks a CU (12 heads of
// 478 x 128 30 -> 26 us, 96 of 82 x 64 x 128 16 -> 12) and loses later (64 of 1000 x 128 100 -> 105); bf16 gains nothing.
// Beside every number of segments between 1 and 64, on 60 calls of random sizes (1 to 128 heads, 32 to 25,000 rows, 20 to 256 wide), forward and backward:
// the choice takes at most 6 % longer than the best in 109 of 120, up to 1.4 times as long in ten, 1.7 times for 16 heads of 21,268, 20 wide.
Plan plan_of(const Problem& pb, int scans, int states) {
  const dark_decay_params& p = pb.p;
  const int C = p.io_dtype == DARK_BF16 ? kChunkBf16 : kChunkF32;
  const int chunks = p.L > 0 ? (p.L + C - 1) / C : 1;
  // scans of both orientations: the larger width counts
  const int d1 = scans > 1 && p.dv > p.dk ? p.dv : p.dk, d2 = scans > 1 && p.dk > p.dv ? p.dk : p.dv;
  const int most = (int)std::min(64LL, std::max(1LL, kMostGroups / pb.BH()));
  Plan best;
  const long long blocks = pb.BH() * ((d2 + 127) / 128);
  best.narrow = d1 > 128 || d2 <= 64 || (p.io_dtype == DARK_F32 && scans * blocks * chunks <= 1280);
  const Cost cost = cost_of(d1, best.narrow ? 64 : d2);
  const float c = p.io_dtype == DARK_BF16 ? cost.bf16 : cost.f32;
  const float heads = (float)(best.narrow ? pb.BH() * ((d2 + 63) / 64) : blocks);
  if (p.sched_segments > 0) {
    best.nseg = std::min(p.sched_segments, std::min(chunks, most));
  } else {
    float least = 0.f;
    for (int s = 1; s <= chunks && s <= most; ++s) {
      const int each = (chunks + s - 1) / s;
      if (s > 1 && (chunks + each - 1) / each != s) continue;   // the same chunks a segment as with fewer
      float rounds = std::ceil(scans * heads * s / 256.f);
      if (rounds == 1.f && scans * heads * s > 192.f && d1 <= 128) rounds = 1.12f;   // with one a CU everywhere, none hides another's waits
      float us = 4.f + each * c * rounds;
      if (s > 1) {
        us += 8.f + each * 0.45f * c * std::ceil(states * heads * (s - 1) / 256.f);
        us += 0.2f * s + 2.f * 4.f * states * (float)pb.BH() * s * p.dk * p.dv / 5.5e6f;
      }
      if (s == 1 || us < least) {
        least = us;
        best.nseg = s;
      }
    }
    if (p.io_dtype == DARK_BF16 && chunks >= 2 && chunks <= 16 && pb.BH() * (chunks + 4) <= kMostGroups) {
      // rows that begin anywhere take registers: past 64 inner values there is room for one workgroup a CU instead of two (the backward pass of
      // 96 heads of 264, 33 and 65 wide: 48 us, as one segment 31)
      const float share = d1 <= 64 || (p.dk % 8 == 0 && p.dv % 8 == 0) ? 1.f : 0.5f;
      const float pairs = scans * heads * (float)(chunks * (chunks + 1) / 2) / (share * cost.pairs), steps = (float)((chunks + 1) / 2) * cost.step;
      if (6.f + (pairs > steps ? pairs : steps) < least) {
        best.direct = true;
        best.nseg = 1;
      }
    }
  }
  const int each = (chunks + best.nseg - 1) / best.nseg;
  best.seg_len = each * C;
  best.nseg = (chunks + each - 1) / each;
  return best;
}
Plan forward_plan(const Problem& pb) { return plan_of(pb, 1, 1); }
Plan backward_plan(const Problem& pb) { return plan_of(pb, 3, 2); }

dark_status run_scan(const Problem& pb, const Plan& plan, const Scans& a, int n) {
  if (plan.direct) return launch_short_bf16(a, n, pb.st);
  return pb.p.io_dtype == DARK_BF16 ? launch_scan_bf16(a, n, pb.st) : launch_scan_f32(a, n, pb.st);
}

// The states before every segment, for `n` states of the same widths.
dark_status run_states(const Problem& pb, const States& a, int n) {
  DARK_TRY(pb.p.io_dtype == DARK_BF16 ? launch_state_bf16(a, n, pb.st) : launch_state_f32(a, n, pb.st));
  const long long size = (long long)a.s[0].d1 * a.s[0].d2;
  if (size % 4 == 0) {
    const dim3 grid((unsigned)pb.BH(), (unsigned)((size / 4 + 255) / 256), n);
    DARK_LAUNCH(KID_DECAY_PREFIX, pb.st, k_decay_prefix<4>, grid, dim3(256), 0, a);
  } else {
    const dim3 grid((unsigned)pb.BH(), (unsigned)((size + 255) / 256), n);
    DARK_LAUNCH(KID_DECAY_PREFIX, pb.st, k_decay_prefix<1>, grid, dim3(256), 0, a);
  }
  return DARK_OK;
}

// Whether the scans of a backward pass, [dv, dk] wide two of them and [dk, dv] the third, are one launch: where the instances are the
// same, and up to 128 wide also where one of them is wider than its scans (bf16, 64 and 128 wide: 4 heads of 500 22 -> 14 us, 96 of them
// 45 -> 41, 32 of 2000 59 -> 58).  fp32 pays for products with zeros as soon as the chip is full: 3 heads of 223 22 -> 19 us, 96 of 82
// 29 -> 35, so there with a workgroup a CU at most.
bool together(const Problem& pb, const Plan& plan) {
  const auto kind = [](int d) { return d > 128 ? 2 : d > 64 ? 1 : 0; };
  const int dk = kind(pb.p.dk), dv = kind(pb.p.dv);
  return dk == dv || (dk < 2 && dv < 2 && (pb.p.io_dtype == DARK_BF16 || 3 * pb.BH() * plan.nseg <= 256));
}

template <typename A>
void fill(const Problem& pb, A& a, const float* log_decay, const int32_t* lengths, const Plan& plan) {
  a.narrow = plan.narrow;
  a.log_decay = log_decay;
  a.lengths = lengths;
  a.B = pb.p.B;
  a.H = pb.p.H;
  a.L = pb.p.L;
  a.layout = pb.p.layout;
  a.nseg = plan.nseg;
  a.seg_len = plan.seg_len;
}

}  // namespace

dark_status forward(const Problem& pb, Arena& ar, const void* Q, const void* K, const void* V, const float* log_decay,
                    const int32_t* lengths, const float* S_in, void* out, float* S_out) {
  const int dk = pb.p.dk, dv = pb.p.dv;
  const Plan plan = forward_plan(pb);
  const int nseg = plan.nseg;
  float* const seg = nseg > 1 ? ar.take<float>((size_t)pb.BH() * nseg * dk * dv) : nullptr;
  if (plan.direct && S_in != nullptr && S_in == S_out) {
    const long long size = pb.BH() * dk * dv;
    float* const copy = ar.take<float>((size_t)size);
    if (ar.overflow) return DARK_EWORKSPACE;
    const long long blocks = (size + 1023) / 1024;
    DARK_LAUNCH(KID_DECAY_COPY, pb.st, k_decay_copy, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, S_in, copy, size);
    S_in = copy;
  }
  if (ar.overflow) return DARK_EWORKSPACE;
  if (nseg > 1) {
    States st;
    fill(pb, st, log_decay, lengths, plan);
    st.s[0] = st.s[1] = State{K, V, S_in, seg, dk, dv, 0, 0, 1.f};
    DARK_TRY(run_states(pb, st, 1));
  }
  Scans a;
  fill(pb, a, log_decay, lengths, plan);
  a.s[0] = a.s[1] = a.s[2] = Scan{Q, K, V, out, nseg > 1 ? seg : S_in, S_out, dk, dv, 0, 0, 0, pb.scale, pb.scale, 1.f};
  return run_scan(pb, plan, a, 1);
}

dark_status backward(const Problem& pb, Arena& ar, const void* Q, const void* K, const void* V, const float* log_decay,
                     const int32_t* lengths, const float* S_in, const void* dOut, const float* dS_out, void* dQ, void* dK,
                     void* dV, float* dS_in) {
  const int dk = pb.p.dk, dv = pb.p.dv;
  const Plan plan = backward_plan(pb);
  const int nseg = plan.nseg;
  const size_t states = (size_t)pb.BH() * nseg * dk * dv;
  float* const sseg = nseg > 1 ? ar.take<float>(states) : nullptr;
  float* const gseg = nseg > 1 ? ar.take<float>(states) : nullptr;
  if (ar.overflow) return DARK_EWORKSPACE;
  const float s = pb.scale;
  const bool rev = dK != nullptr || dV != nullptr || dS_in != nullptr;
  if (nseg > 1) {
    States st;
    fill(pb, st, log_decay, lengths, plan);
    int n = 0;
    if (dQ != nullptr) st.s[n++] = State{K, V, S_in, sseg, dk, dv, 0, 0, 1.f};
    if (rev) st.s[n++] = State{Q, dOut, dS_out, gseg, dk, dv, 1, 1, s};
    if (n == 1) st.s[1] = st.s[0];
    if (n > 0) DARK_TRY(run_states(pb, st, n));
  }
  const float* const Su = nseg > 1 ? sseg : S_in;
  const float* const Gu = nseg > 1 ? gseg : dS_out;
  const Scan q{dOut, V, K, dQ, Su, nullptr, dv, dk, 1, 0, 0, s, s, 1.f};
  const Scan k{V, dOut, Q, dK, Gu, nullptr, dv, dk, 1, 1, 1, s, 1.f, s};
  const Scan v{K, Q, dOut, dV, Gu, dS_in, dk, dv, 0, 1, 1, s, 1.f, s};
  Scans a;
  fill(pb, a, log_decay, lengths, plan);
  int n = 0;
  if (dQ != nullptr) a.s[n++] = q;
  if (dK != nullptr) a.s[n++] = k;
  if (n > 0 && !together(pb, plan)) {   // dV has other widths: a launch of its own
    for (int i = n; i < kMostScans; ++i) a.s[i] = a.s[0];
    DARK_TRY(run_scan(pb, plan, a, n));
    n = 0;
  }
  if (dV != nullptr || dS_in != nullptr) a.s[n++] = v;
  if (n == 0) return DARK_OK;
  for (int i = n; i < kMostScans; ++i) a.s[i] = a.s[0];
  return run_scan(pb, plan, a, n);
}

dark_status step(const Problem& pb, const void* q, const void* k, const void* v, const float* log_decay, const int32_t* parent,
                 int state_rows, const float* S_in, float* S_out, void* out) {
  const int dk = pb.p.dk, dv = pb.p.dv, H = pb.p.H;
  const int W = dv % 4 == 0 ? 4 : 1, units = (dv + W - 1) / W;
  // Columns of a workgroup: all of them, or fewer (16 at least, 64 bytes of a row) until there are four workgroups a CU.
  int tx = 1;
  while (tx < units) tx *= 2;
  const int least = 16 / W;
  while (tx > least && pb.BH() * ((units + tx - 1) / tx) < 1024) tx /= 2;
  const dim3 grid((unsigned)pb.BH(), (unsigned)((units + tx - 1) / tx));
#define DARK_STEP(T, WW)                                                                                                        \
  DARK_LAUNCH(KID_DECAY_STEP, pb.st, (k_decay_step<T, WW>), grid, dim3(256), 0, static_cast<const T*>(q), static_cast<const T*>(k), \
              static_cast<const T*>(v), log_decay, parent, state_rows, S_in, S_out, static_cast<T*>(out), H, dk, dv, tx, pb.scale)
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

}  // namespace decay
}  // namespace dark

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------
using namespace dark;

namespace {
size_t size_of(const dark_decay_params& p) { return p.io_dtype == DARK_BF16 ? 2 : 4; }
// Bytes of Q or K, of V, of a state.
struct Sizes {
  size_t k, v, state, decay, lengths;
  explicit Sizes(const decay::Problem& pb) {
    const size_t rows = (size_t)pb.BH() * pb.p.L * size_of(pb.p);
    k = rows * pb.p.dk;
    v = rows * pb.p.dv;
    state = (size_t)pb.BH() * pb.p.dk * pb.p.dv * sizeof(float);
    decay = (size_t)pb.p.H * sizeof(float);
    lengths = (size_t)pb.p.B * sizeof(int32_t);
  }
};
dark_status check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return DARK_OK;
  if (ws == nullptr || ws_bytes < need) return DARK_EWORKSPACE;
  return aligned(ws, 256) ? DARK_OK : DARK_EALIGN;
}
// `in_place`: the forward call updates a state in place, or may.
size_t measure(const decay::Problem& pb, bool bwd, bool in_place) {
  const decay::Plan plan = bwd ? decay::backward_plan(pb) : decay::forward_plan(pb);
  Arena ar(nullptr, 0);
  const size_t state = (size_t)pb.BH() * pb.p.dk * pb.p.dv;
  if (plan.direct && !bwd && in_place) (void)ar.take<float>(state);
  for (int i = 0; plan.nseg > 1 && i < (bwd ? 2 : 1); ++i) (void)ar.take<float>(state * plan.nseg);
  return ar.off;
}
}  // namespace

extern "C" {

size_t dark_decay_workspace_bytes(const dark_decay_params* p, int backward) {
  decay::Problem pb;
  if (decay::check_params(p, &pb) != DARK_OK || pb.p.B == 0) return 0;
  return measure(pb, backward != 0, true);
}

dark_status dark_decay_fwd(const dark_decay_params* p, const void* Q, const void* K, const void* V, const float* log_decay,
                           const int32_t* lengths, const float* S_in, void* out, float* S_out, void* ws, size_t ws_bytes,
                           void* hip_stream) {
  decay::Problem pb;
  DARK_TRY(decay::check_params(p, &pb));
  if (pb.p.B == 0 || (pb.p.L == 0 && S_out == nullptr)) return DARK_OK;
  if (log_decay == nullptr) return DARK_EINVAL;
  if (pb.p.L > 0 && (!Q || !K || !V || !out)) return DARK_EINVAL;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(S_in, 16) || !aligned(S_out, 16) ||
      !aligned(log_decay, 4) || !aligned(lengths, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  if (S_in != S_out && overlap({S_in, n.state}, {S_out, n.state})) return DARK_EINVAL;
  const size_t need = measure(pb, false, S_in != nullptr && S_in == S_out);
  DARK_TRY(check_workspace(ws, ws_bytes, need));
  if (overlap({{out, n.v}, {S_out, n.state}}, {{Q, n.k}, {K, n.k}, {V, n.v}, {log_decay, n.decay}, {lengths, n.lengths}}) ||
      overlap({out, n.v}, {S_in, n.state}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  Arena ar(ws, ws_bytes);
  return decay::forward(pb, ar, Q, K, V, log_decay, lengths, S_in, out, S_out);
}

dark_status dark_decay_bwd(const dark_decay_params* p, const void* Q, const void* K, const void* V, const float* log_decay,
                           const int32_t* lengths, const float* S_in, const void* dOut, const float* dS_out, void* dQ, void* dK,
                           void* dV, float* dS_in, void* ws, size_t ws_bytes, void* hip_stream) {
  decay::Problem pb;
  DARK_TRY(decay::check_params(p, &pb));
  if (pb.p.B == 0 || (pb.p.L == 0 && dS_in == nullptr)) return DARK_OK;
  if (log_decay == nullptr) return DARK_EINVAL;
  if (pb.p.L > 0 && (!Q || !K || !V || !dOut)) return DARK_EINVAL;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(dOut, 16) || !aligned(S_in, 16) || !aligned(dS_out, 16) ||
      !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16) || !aligned(dS_in, 16) || !aligned(log_decay, 4) || !aligned(lengths, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  if (overlap({dS_in, n.state}, {dS_out, n.state}) || overlap({dS_in, n.state}, {S_in, n.state})) return DARK_EINVAL;
  const size_t need = measure(pb, true, false);
  DARK_TRY(check_workspace(ws, ws_bytes, need));
  if (overlap({{dQ, n.k}, {dK, n.k}, {dV, n.v}, {dS_in, n.state}}, {{Q, n.k}, {K, n.k}, {V, n.v}, {dOut, n.v}, {S_in, n.state}, {dS_out, n.state},
                                                                    {log_decay, n.decay}, {lengths, n.lengths}}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  Arena ar(ws, ws_bytes);
  return decay::backward(pb, ar, Q, K, V, log_decay, lengths, S_in, dOut, dS_out, dQ, dK, dV, dS_in);
}

dark_status dark_decay_step(const dark_decay_params* p, const void* q, const void* k, const void* v, const float* log_decay,
                            const int32_t* parent, int state_rows, const float* S_in, float* S_out, void* out, void* hip_stream) {
  decay::Problem pb;
  DARK_TRY(decay::check_params(p, &pb));
  pb.p.L = 1;
  if (pb.p.B == 0) return DARK_OK;
  if (!q || !k || !v || !log_decay || !S_in || !S_out || !out) return DARK_EINVAL;
  if (parent == nullptr ? state_rows != pb.p.B : state_rows <= 0) return DARK_EINVAL;
  const size_t elem = size_of(pb.p);   // rows of one tensor, slices of a longer one: no more is asked of them
  if (!aligned(q, elem) || !aligned(k, elem) || !aligned(v, elem) || !aligned(out, elem) || !aligned(S_in, 16) || !aligned(S_out, 16) ||
      !aligned(log_decay, 4) || !aligned(parent, 4))
    return DARK_EALIGN;
  const Sizes n(pb);
  const size_t past = n.state / pb.p.B * state_rows;
  if ((parent != nullptr || S_in != S_out) && overlap({S_in, past}, {S_out, n.state})) return DARK_EINVAL;
  if (overlap({{out, n.v}, {S_out, n.state}}, {{q, n.k}, {k, n.k}, {v, n.v}, {log_decay, n.decay}, {parent, n.lengths}}) ||
      overlap({out, n.v}, {S_in, past}))
    return DARK_EINVAL;
  pb.st = static_cast<hipStream_t>(hip_stream);
  return decay::step(pb, q, k, v, log_decay, parent, state_rows, S_in, S_out, out);
}

}  // extern "C"
