// Beam search over recurrent states: the selection of the next beams from their logits, and the reordering of the states that
// belong to them.
//
// Selection, per batch entry with n beams: candidate (j, t) is worth score_j + logit_jt - log sum_u exp logit_ju; the n largest win,
// equal ones by the lowest j, then the lowest t.  k_beam_rows reads every logit once: a workgroup takes a slice of a row and leaves
// the slice's maximum, its sum of exponentials and, wave by wave, the n largest logits in order.  k_beam_pick joins the sums of a
// batch entry's rows and merges the sorted lists from their heads.  Bound by reading the logits; few rows are cut into more slices.
// Two candidates of different beams may lie closer together than fp32 resolves: offsets and comparisons are in fp64.
#include <cmath>

#include "common.h"

namespace dark {
namespace beam {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

struct Entry {
  float logit;
  int token;
};
struct Part {
  float top, sum;
};

// Monotone in the value for everything but NaN, which the callers replace; 0 is below every value.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

__device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : v == 0.f ? 0.f : v; }   // one zero

// Largest key of the wave.
template <int CTRL>
__device__ __forceinline__ unsigned dpp_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
  return o > v ? o : v;
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  v = dpp_max<0x121>(v);   // rotations within a row of 16 lanes by 1, 2, 4, 8
  v = dpp_max<0x122>(v);
  v = dpp_max<0x124>(v);
  v = dpp_max<0x128>(v);
  const unsigned a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16), c = __builtin_amdgcn_readlane(v, 32),
                 d = __builtin_amdgcn_readlane(v, 48);
  const unsigned ab = a > b ? a : b, cd = c > d ? c : d;
  return ab > cd ? ab : cd;
}

// A score that is no number, or infinite, leaves its beam without candidates: whatever is compared below is a number or -infinity.
__device__ __forceinline__ bool finite(float v) { return v > -INFINITY && v < INFINITY; }

constexpr int kMostBeams = 32;

// A slice is 256 E elements of a row; thread t holds pieces t, t + 256, ... of 16 bytes.  Rows begin where they begin: the slices
// count from the 16-byte boundary at or before the row's first element.
template <typename T, int E>
__global__ __launch_bounds__(256) void k_beam_rows(const T* __restrict__ logits, const float* __restrict__ scores,
                                                   const unsigned char* __restrict__ finished, Part* __restrict__ parts,
                                                   Entry* __restrict__ lists, int n, int V, long long total) {
  constexpr int P = 16 / (int)sizeof(T), N = E / P;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, slice = blockIdx.x, slices = gridDim.x, row = blockIdx.y;
  if ((finished != nullptr && finished[row] != 0) || !finite(scores[row])) return;   // k_beam_pick knows what these offer
  const long long first = (long long)row * V, base = first / P * P + (long long)slice * 256 * E;
  unsigned key[E];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const long long at = base + (long long)(i * 256 + tid) * P;
    T v[P];
    if (at + P <= total) {
      const u32x4 r = *reinterpret_cast<const u32x4*>(logits + at);
      __builtin_memcpy(v, &r, 16);
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j) v[j] = at + j < total ? logits[at + j] : (T)0;
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float f;
      if constexpr (sizeof(T) == 2) f = __uint_as_float((unsigned)v[j] << 16);
      else f = v[j];
      const long long t = at + j - first;
      key[i * P + j] = t >= 0 && t < V ? ordered(clean(f)) : 0u;
    }
  }
  // maximum and sum of exponentials
  unsigned best = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) best = key[e] > best ? key[e] : best;
  __shared__ unsigned tops[4];
  __shared__ float sums[4];
  const unsigned wtop = wave_max(best);
  if (lane == 0) tops[wave] = wtop;
  __syncthreads();
  unsigned top = tops[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) top = tops[i] > top ? tops[i] : top;
  const float m = top != 0 ? value_of(top) : -INFINITY;
  float s = 0.f;
  if (finite(m)) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      // exp(x) = 2^(x log2 e) with the product's rounding error made good: far below the maximum it would be 2^-20 of the term
      const float x = key[e] != 0 ? value_of(key[e]) - m : -INFINITY, t = x * 1.4426950408889634f;
      const float low = fmaf(x, 1.4426950408889634f, -t) + x * 1.925963033500234e-8f;
      const float p = __builtin_amdgcn_exp2f(t);
      s += p > 0.f ? fmaf(p, 0.6931471805599453f * low, p) : 0.f;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) sums[wave] = s;
  __syncthreads();
  if (tid == 0) parts[(long long)row * slices + slice] = Part{m, (sums[0] + sums[1]) + (sums[2] + sums[3])};
  // the wave's n largest, in order
  Entry* const list = lists + (((long long)row * slices + slice) * 4 + wave) * n;
  unsigned mine = best;
  for (int i = 0; i < n; ++i) {
    const unsigned w = wave_max(mine);
    if (w == 0) {   // no values left: token -1 ends the list
      if (lane == 0) list[i] = Entry{0.f, -1};
      break;
    }
    int at = 0x7fffffff;   // the lane's first element of that value
    if (mine == w) {
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (key[e] == w) at = e;
    }
    long long t = at != 0x7fffffff ? base - first + (long long)(at / P * 256 + tid) * P + at % P : 0x7fffffff;
    int token = (int)t;
    u64 has = __ballot(mine == w);
    int low;
    if ((has & (has - 1)) == 0) {
      low = __builtin_amdgcn_readlane(token, __builtin_ctzll(has));
    } else {
      low = token;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) low = min(low, __shfl_xor(low, o, 64));
    }
    if (token == low && mine == w) {
      list[i] = Entry{value_of(w), low};
      unsigned next = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        key[e] = e == at ? 0u : key[e];
        next = key[e] > next ? key[e] : next;
      }
      mine = next;
    }
  }
}

// ---------------------------------------------------------------------------
// One workgroup a batch entry.  List l of the n * slices * 4 belongs to beam l / (4 slices); thread t watches over lists t, t + 256, ...
// ---------------------------------------------------------------------------
constexpr int kMostLists = 32768;

struct Head {
  double value;
  unsigned flat;   // beam * V + token; ~0: none
};
__device__ __forceinline__ bool before(const Head& a, const Head& b) { return a.value > b.value || (a.value == b.value && a.flat < b.flat); }

enum { kAlive = 0, kFinished = 1, kDead = 2 };

__global__ __launch_bounds__(256) void k_beam_pick(const Part* __restrict__ parts, const Entry* __restrict__ lists,
                                                   const float* __restrict__ scores, const unsigned char* __restrict__ finished, int n,
                                                   int V, int slices, int eos, int keep_slots, float* __restrict__ out_scores,
                                                   int32_t* __restrict__ out_parent, int32_t* __restrict__ out_token) {
  extern __shared__ __attribute__((aligned(16))) unsigned char taken[];   // entries taken from every list
  __shared__ double offset[kMostBeams];
  __shared__ int kind[kMostBeams];
  __shared__ double wv[4];
  __shared__ unsigned wf[4];
  __shared__ double pick_value[kMostBeams];
  __shared__ unsigned pick_flat[kMostBeams];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x, per = 4 * slices, count = n * per;
  for (int l = tid; l < count; l += 256) taken[l] = 0;
  for (int j = wave; j < n; j += 4) {
    const long long row = (long long)b * n + j;
    const float score = scores[row];
    if (finished != nullptr && finished[row] != 0) {
      if (lane == 0) {
        kind[j] = kFinished;
        offset[j] = finite(score) ? (double)score : -INFINITY;
      }
      continue;
    }
    double z = 0.0;
    float top = -INFINITY;
    if (finite(score)) {
      for (int i = lane; i < slices; i += 64) top = fmaxf(top, parts[row * slices + i].top);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      for (int i = lane; i < slices; i += 64) {
        const Part p = parts[row * slices + i];
        if (p.sum > 0.f) z += (double)p.sum * exp((double)p.top - (double)top);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
    }
    if (lane == 0) {
      const bool alive = finite(top);
      kind[j] = alive ? kAlive : kDead;
      offset[j] = alive ? (double)score - ((double)top + log(z)) : -INFINITY;
    }
  }
  __syncthreads();
  const Entry* const own = lists + (long long)b * count * n;
  // what list l offers after `at` of its entries
  const auto head = [&](int l, int at) {
    const int j = l / per;
    Head hd{-INFINITY, ~0u};
    if (kind[j] == kAlive) {
      if (at >= n) return hd;
      const Entry e = own[(long long)l * n + at];
      if (e.token < 0) return hd;
      hd.value = offset[j] + (double)e.logit;
      hd.flat = (unsigned)j * (unsigned)V + (unsigned)e.token;
    } else if (l % per == 0 && at < V) {   // a finished beam goes on with `eos` alone; what else it and a dead one offer is worth nothing
      int token = at;
      if (kind[j] == kFinished) {
        token = at == 0 ? eos : at - 1 + (at - 1 >= eos ? 1 : 0);
        if (at == 0) hd.value = offset[j];
      }
      hd.flat = (unsigned)j * (unsigned)V + (unsigned)token;
    }
    return hd;
  };
  Head mine{-INFINITY, ~0u};
  int from = -1;
  const auto rescan = [&]() {
    mine = Head{-INFINITY, ~0u};
    from = -1;
    for (int l = tid; l < count; l += 256) {
      const Head hd = head(l, taken[l]);
      if (hd.flat != ~0u && (from < 0 || before(hd, mine))) {
        mine = hd;
        from = l;
      }
    }
  };
  rescan();
  for (int i = 0; i < n; ++i) {
    Head w = mine;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      Head x;
      x.value = __shfl_xor(w.value, o, 64);
      x.flat = __shfl_xor(w.flat, o, 64);
      if (before(x, w)) w = x;
    }
    if (lane == 0) {
      wv[wave] = w.value;
      wf[wave] = w.flat;
    }
    __syncthreads();
    w = Head{wv[0], wf[0]};
#pragma unroll
    for (int k = 1; k < 4; ++k)
      if (before(Head{wv[k], wf[k]}, w)) w = Head{wv[k], wf[k]};
    if (tid == 0) {
      pick_value[i] = w.value;
      pick_flat[i] = w.flat;
    }
    if (from >= 0 && mine.flat == w.flat) {
      ++taken[from];
      rescan();
    }
    __syncthreads();
  }
  if (tid == 0) {
    unsigned used = 0;   // slots that are given away
    if (keep_slots) {
      for (int i = 0; i < n; ++i) used |= 1u << (pick_flat[i] / (unsigned)V);
    }
    unsigned kept = 0;
    int free = 0;
    for (int i = 0; i < n; ++i) {
      const int parent = (int)(pick_flat[i] / (unsigned)V), token = (int)(pick_flat[i] % (unsigned)V);
      int slot = i;
      if (keep_slots) {
        if ((kept >> parent & 1u) == 0) {
          kept |= 1u << parent;
          slot = parent;
        } else {
          while (used >> free & 1u) ++free;
          slot = free++;
        }
      }
      const long long at = (long long)b * n + slot;
      out_scores[at] = (float)pick_value[i];
      out_parent[at] = parent;
      out_token[at] = token;
    }
  }
}

// ---------------------------------------------------------------------------
// States in place: a thread holds the same 16 (4, 1) bytes of every row that changes, so that all are read before any is written.
// Bound by reading the parents of the rows that change and writing those rows.
// ---------------------------------------------------------------------------
constexpr int kMostTensors = 16;
struct Tensors {
  char* data[kMostTensors];
  long long row_bytes[kMostTensors];
  int unit[kMostTensors];          // 16, 4 or 1
  int first[kMostTensors + 1];     // blocks before the tensor's own
  int count;
};

template <typename U, int N>
__device__ __forceinline__ void reorder(char* rows, long long row_bytes, long long at, const int32_t* from, int n) {
  U v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (j < n) {
      const int p = from[j];
      if (p != j && (unsigned)p < (unsigned)n) v[j] = *reinterpret_cast<const U*>(rows + p * row_bytes + at);
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (j < n) {
      const int p = from[j];
      if (p != j && (unsigned)p < (unsigned)n) *reinterpret_cast<U*>(rows + j * row_bytes + at) = v[j];
    }
  }
}

template <int N>
__global__ __launch_bounds__(256) void k_state_reorder(Tensors t, const int32_t* __restrict__ parent, int n) {
  int i = 0;
  while (i + 1 < t.count && (int)blockIdx.x >= t.first[i + 1]) ++i;
  const long long at = ((long long)((int)blockIdx.x - t.first[i]) * 256 + threadIdx.x) * t.unit[i], row_bytes = t.row_bytes[i];
  if (at >= row_bytes) return;
  char* const rows = t.data[i] + (long long)blockIdx.y * n * row_bytes;
  const int32_t* const from = parent + (long long)blockIdx.y * n;
  if (t.unit[i] == 16) reorder<u32x4, N>(rows, row_bytes, at, from, n);
  else if (t.unit[i] == 4) reorder<unsigned, N>(rows, row_bytes, at, from, n);
  else reorder<unsigned char, N>(rows, row_bytes, at, from, n);
}

// Elements a thread holds: 32, or 8 where the rows are too few to give every CU a workgroup.
int slice_elements(const dark_beam_params& p) {
  const long long rows = (long long)p.B * p.n;
  return rows * ((p.V + 8191) / 8192) >= 512 ? 32 : 8;
}
int slices_of(const dark_beam_params& p) {
  const int per = p.io_dtype == DARK_BF16 ? 8 : 4, len = 256 * slice_elements(p);
  return (int)(((long long)p.V + per - 1 + len - 1) / len);   // a row begins up to per - 1 elements behind its first slice
}

dark_status check(const dark_beam_params* p) {
  if (p == nullptr || p->B < 0 || p->n <= 0 || p->V <= 0) return DARK_EINVAL;
  if (p->io_dtype != DARK_F32 && p->io_dtype != DARK_BF16) return DARK_EINVAL;
  if (p->n > kMostBeams || (long long)p->n * p->V >= (1LL << 31) || (long long)p->B * p->n > 65535) return DARK_EUNSUPPORTED;
  if ((long long)p->n * 4 * slices_of(*p) > kMostLists) return DARK_EUNSUPPORTED;
  return DARK_OK;
}

void plan(const dark_beam_params& p, Arena& ar, Part** parts, Entry** lists) {
  const size_t slots = (size_t)p.B * p.n * slices_of(p);
  *parts = ar.take<Part>(slots);
  *lists = ar.take<Entry>(slots * 4 * p.n);
}

template <typename T>
dark_status rows(const dark_beam_params& p, const void* logits, const float* scores, const unsigned char* finished, Part* parts,
                 Entry* lists, hipStream_t st) {
  const dim3 grid(slices_of(p), p.B * p.n);
  const long long total = (long long)p.B * p.n * p.V;
  if (slice_elements(p) == 32) {
    DARK_LAUNCH(KID_BEAM_ROWS, st, (k_beam_rows<T, 32>), grid, dim3(256), 0, static_cast<const T*>(logits), scores, finished, parts, lists, p.n, p.V, total);
  } else {
    DARK_LAUNCH(KID_BEAM_ROWS, st, (k_beam_rows<T, 8>), grid, dim3(256), 0, static_cast<const T*>(logits), scores, finished, parts, lists, p.n, p.V, total);
  }
  return DARK_OK;
}

}  // namespace
}  // namespace beam
}  // namespace dark

using namespace dark;

extern "C" {

size_t dark_beam_workspace_bytes(const dark_beam_params* p) {
  if (beam::check(p) != DARK_OK || p->B == 0) return 0;
  Arena ar(nullptr, 0);
  beam::Part* parts;
  beam::Entry* lists;
  beam::plan(*p, ar, &parts, &lists);
  return ar.off;
}

dark_status dark_beam_select(const dark_beam_params* p, const void* logits, const float* scores, const unsigned char* finished,
                             float* out_scores, int32_t* out_parent, int32_t* out_token, void* ws, size_t ws_bytes, void* hip_stream) {
  DARK_TRY(beam::check(p));
  if (p->B == 0) return DARK_OK;
  if (!logits || !scores || !out_scores || !out_parent || !out_token) return DARK_EINVAL;
  if (finished != nullptr && (p->eos < 0 || p->eos >= p->V)) return DARK_EINVAL;
  if (!aligned(logits, 16) || !aligned(scores, 4) || !aligned(out_scores, 4) || !aligned(out_parent, 4) || !aligned(out_token, 4))
    return DARK_EALIGN;
  Arena ar(ws, ws_bytes);
  if (ws == nullptr || ws_bytes < dark_beam_workspace_bytes(p)) return DARK_EWORKSPACE;
  if (!aligned(ws, 256)) return DARK_EALIGN;
  beam::Part* parts;
  beam::Entry* lists;
  beam::plan(*p, ar, &parts, &lists);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  DARK_TRY(p->io_dtype == DARK_BF16 ? beam::rows<unsigned short>(*p, logits, scores, finished, parts, lists, st)
                                    : beam::rows<float>(*p, logits, scores, finished, parts, lists, st));
  const int slices = beam::slices_of(*p);
  DARK_LAUNCH(KID_BEAM_PICK, st, beam::k_beam_pick, dim3(p->B), dim3(256), (size_t)p->n * 4 * slices, parts, lists, scores, finished, p->n, p->V,
              slices, p->eos, p->keep_slots != 0, out_scores, out_parent, out_token);
  return DARK_OK;
}

dark_status dark_state_reorder(int B, int n, const int32_t* parent, int count, void* const* states, const size_t* row_bytes,
                               void* hip_stream) {
  if (B < 0 || n <= 0 || count < 0) return DARK_EINVAL;
  if (n > beam::kMostBeams || B > 65535) return DARK_EUNSUPPORTED;
  if (B == 0 || count == 0) return DARK_OK;
  if (parent == nullptr || states == nullptr || row_bytes == nullptr) return DARK_EINVAL;
  if (!aligned(parent, 4)) return DARK_EALIGN;
  for (int i = 0; i < count; ++i) {
    if (row_bytes[i] == 0) continue;
    if (states[i] == nullptr) return DARK_EINVAL;
    if (row_bytes[i] > ((size_t)1 << 38)) return DARK_EUNSUPPORTED;
    if (!aligned(states[i], 16)) return DARK_EALIGN;
  }
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  for (int i = 0; i < count;) {
    beam::Tensors t;
    t.count = 0;
    long long blocks = 0;
    for (; i < count && t.count < beam::kMostTensors; ++i) {
      if (row_bytes[i] == 0) continue;
      const int unit = row_bytes[i] % 16 == 0 ? 16 : row_bytes[i] % 4 == 0 ? 4 : 1;
      const long long more = (long long)((row_bytes[i] / unit + 255) / 256);
      if (blocks + more > (1 << 23)) {
        if (t.count == 0) return DARK_EUNSUPPORTED;
        break;
      }
      t.data[t.count] = static_cast<char*>(states[i]);
      t.row_bytes[t.count] = (long long)row_bytes[i];
      t.unit[t.count] = unit;
      t.first[t.count] = (int)blocks;
      blocks += more;
      ++t.count;
    }
    if (t.count == 0) break;
    t.first[t.count] = (int)blocks;
    const dim3 grid((unsigned)blocks, (unsigned)B);
    if (n <= 4) {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<4>, grid, dim3(256), 0, t, parent, n);
    } else if (n <= 8) {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<8>, grid, dim3(256), 0, t, parent, n);
    } else {
      DARK_LAUNCH(KID_STATE_REORDER, st, beam::k_state_reorder<32>, grid, dim3(256), 0, t, parent, n);
    }
  }
  return DARK_OK;
}

}  // extern "C"
