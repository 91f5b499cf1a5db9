// Calls that move whole fp32 states, with a decay for each head: one token of every sequence, where a sequence may go on
// from another one's state (beams), and the accepted path of a tree of drafted tokens.
//
// Both are a stream of the states through the chip; the arithmetic is fp32 on the vector ALU.  A workgroup owns COLS value
// columns of one state: a row is covered by COLS / 4 lanes with four columns each, and all rows are requested before any is
// used.  128 x 128, bf16 rows: 4096 states with beams 81 us (268 MB written, at most as much read), the same accepted of trees
// of 32 tokens, one sequence in eight rejecting all, 88 us, 5.4 TB/s; 16 states 3.0 and 4.0 us, of which an empty kernel takes
// 2.4.
#include "device_common.h"
#include "launch.h"
#include "tile_io.h"
#include "decay.h"

namespace cottn {
using namespace COTTN_NS;
namespace {

template <typename T> struct Element {
  typedef __attribute__((ext_vector_type(4))) T vec4;
  static __device__ __forceinline__ f32x4 load4(const T* p) {
    const vec4 x = *reinterpret_cast<const vec4*>(p);
    return f32x4{float(x[0]), float(x[1]), float(x[2]), float(x[3])};
  }
};

__device__ __forceinline__ f32x4 load_state4(const float* p, bool stream) {
  return stream ? __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)) : *reinterpret_cast<const f32x4*>(p);
}
__device__ __forceinline__ void store_state4(float* p, f32x4 x) {
  __builtin_nontemporal_store(x, reinterpret_cast<f32x4*>(p));
}

// Row x of D elements normalised by a whole wave, times `factor`; the lane's elements are l and l + 64.
template <typename T, int D>
struct WaveRow {
  float x0, x1;
  __device__ __forceinline__ WaveRow(const T* x, int l) {
    x0 = float(x[l % D]);
    x1 = D > 64 ? float(x[(l + 64) % D]) : 0.f;
  }
  __device__ __forceinline__ void store(float* to, float factor, float eps, int l) {
    const float sum = group_sum<64>(l < D ? x0 * x0 + x1 * x1 : 0.f), f = factor * inv_norm(sum, eps);
    if (l < D) to[l] = f * x0;
    if (D > 64) to[l + 64] = f * x1;
  }
};

template <int DK, int COLS>
struct StateRows {
  static constexpr int TPR = COLS / 4, RPP = 256 / TPR, PASSES = (DK + RPP - 1) / RPP;
  static constexpr bool WHOLE = DK % RPP == 0;
};

// S <- g S_from + kh^T v, o = s qh S with the new S.  parent == null: from the sequence's own place in `from`; else from
// that of sequence parent[b] of `from`, and from nothing where that is none of its n_from.
template <typename T, int DK, int DV, int COLS>
__global__ __launch_bounds__(256) void step_decay_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ s,
    const float* __restrict__ log_decay, const float* from, const int* __restrict__ parent, float* to, T* __restrict__ o,
    Divisor H, int n_from, float eps, int stream) {
  using R = StateRows<DK, COLS>;
  constexpr int PARTS = DV / COLS;
  __shared__ __attribute__((aligned(16))) float qh[DK], kh[DK];
  __shared__ __attribute__((aligned(16))) float partial[R::RPP][COLS];
  fetch_argument_now(q, k, v, s, log_decay, from, parent, to, o, H, n_from, eps, stream);
  const int unit = blockIdx.x / PARTS, part = blockIdx.x % PARTS, b = quotient(unit, H), head = unit - b * H.n;
  const int tid = threadIdx.x, w = tid / 64, l = tid % 64;
  const int col = part * COLS + tid % R::TPR * 4, row0 = tid / R::TPR;
  int src = b;
  if (parent != nullptr) src = parent[b];
  const bool none = src < 0 || src >= n_from;
  const float* S = from + (size_t(none ? 0 : src) * H.n + head) * DK * DV;
  f32x4 rows[R::PASSES];
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    rows[p] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!none && (R::WHOLE || row < DK)) rows[p] = load_state4(S + size_t(row) * DV + col, stream != 0);
  }
  if (w < 2) {
    WaveRow<T, DK> x((w == 0 ? q : k) + size_t(unit) * DK, l);
    x.store(w == 0 ? qh : kh, 1.f, eps, l);
  }
  const f32x4 v4 = Element<T>::load4(v + size_t(unit) * DV + col);
  const float scale = s[head];
  const Kept kept(Decay(log_decay != nullptr ? log_decay[head] : 0.f), 1.f);
  __syncthreads();
  float* out = to + size_t(unit) * DK * DV;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    if (R::WHOLE || row < DK) {
      const float kr = kh[row], qr = qh[row];
      f32x4 x = kept.of(rows[p]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = __builtin_fmaf(kr, v4[i], x[i]);
        acc[i] = __builtin_fmaf(qr, x[i], acc[i]);
      }
      store_state4(out + size_t(row) * DV + col, x);
    }
  }
  *reinterpret_cast<f32x4*>(&partial[row0][tid % R::TPR * 4]) = acc;
  __syncthreads();
  if (tid < COLS) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < R::RPP; ++i) sum += partial[i][tid];
    o[size_t(unit) * DV + part * COLS + tid] = static_cast<T>(scale * sum);
  }
}

// S <- g^L S + sum over the L tokens j of the path to node `last` of g^(L-1-depth_j) kh_j^T v_j; last outside the tree: S
// stays.
template <typename T, int DK, int DV, int COLS>
__global__ __launch_bounds__(256) void tree_accept_kernel(
    const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ log_decay, const int* __restrict__ parent,
    const int* __restrict__ last, float* __restrict__ state, Divisor H, int n_tokens, float eps, int stream) {
  using R = StateRows<DK, COLS>;
  constexpr int PARTS = DV / COLS, MOST = 16;   // path tokens at a time
  __shared__ __attribute__((aligned(16))) float kw[MOST][DK];
  __shared__ __attribute__((aligned(16))) float vs[MOST][COLS];
  fetch_argument_now(k, v, log_decay, parent, last, state, H, n_tokens, eps, stream);
  const int unit = blockIdx.x / PARTS, part = blockIdx.x % PARTS, b = quotient(unit, H), head = unit - b * H.n;
  const int end = last[b];
  if (end < 0 || end >= n_tokens) return;
  const int tid = threadIdx.x, w = tid / 64, l = tid % 64;
  const int col = part * COLS + tid % R::TPR * 4, row0 = tid / R::TPR;
  float* S = state + size_t(unit) * DK * DV;
  f32x4 rows[R::PASSES];
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    rows[p] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (R::WHOLE || row < DK) rows[p] = load_state4(S + size_t(row) * DV + col, stream != 0);
  }
  const Decay g(log_decay != nullptr ? log_decay[head] : 0.f);
  unsigned long long path = __shfl(TreeNode(parent + size_t(b) * n_tokens, n_tokens, l).path, end, 64);
  path = (static_cast<unsigned long long>(unsigned(__builtin_amdgcn_readfirstlane(int(path >> 32)))) << 32) |
         unsigned(__builtin_amdgcn_readfirstlane(int(path)));
  const int length = __builtin_popcountll(path);
  const Kept kept(g, float(length));
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) rows[p] = kept.of(rows[p]);
  for (int first = 0; first < length; first += MOST) {
    const int n = min(MOST, length - first);
    // wave w takes every fourth token of the path
    unsigned long long rest = path;
    for (int m = 0; m < n; ++m) {
      const int j = __builtin_ctzll(rest);
      rest &= rest - 1;
      if (m % 4 != w) continue;
      const size_t at = size_t(unit) * n_tokens + j;
      WaveRow<T, DK> x(k + at * DK, l);
      x.store(kw[m], g.after(float(length - 1 - first - m)), eps, l);
      if (l < COLS) vs[m][l] = float(v[at * DV + part * COLS + l]);
      if (COLS > 64) vs[m][(l + 64) % COLS] = float(v[at * DV + part * COLS + (l + 64) % COLS]);
    }
    path = rest;
    __syncthreads();
    for (int m = 0; m < n; ++m) {
      const f32x4 v4 = *reinterpret_cast<const f32x4*>(&vs[m][tid % R::TPR * 4]);
#pragma unroll
      for (int p = 0; p < R::PASSES; ++p) {
        const int row = p * R::RPP + row0;
        if (R::WHOLE || row < DK) {
#pragma unroll
          for (int i = 0; i < 4; ++i) rows[p][i] = __builtin_fmaf(kw[m][row], v4[i], rows[p][i]);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    if (R::WHOLE || row < DK) store_state4(S + size_t(row) * DV + col, rows[p]);
  }
}

// non-temporal loads where the states of a call exceed the L2s (step.hip)
bool streamed(long units, int dk, int dv) { return double(units) * dk * dv * sizeof(float) > 32.0 * 1024 * 1024; }

// Up to 128 states a workgroup takes 32 value columns instead of all, so that more compute units have one.  Kernels alone,
// states of 128 x 128, whole / parts: step of 16 states 3.6 / 3.0 us, 128 5.4 / 4.2, 256 6.9 / 7.9; accepting 5.2 / 4.0, 7.5 /
// 5.2, 8.7 / 8.9.
bool state_parts(long units, int dv) { return dv > 32 && units <= 128; }

template <typename T, int DK, int DV, int COLS>
hipError_t step_parts(const StepDecayArgs& a) {
  const int units = a.B * a.H;
  return launch_kernel("step_decay_kernel", step_decay_kernel<T, DK, DV, COLS>, dim3(units * (DV / COLS)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.q), static_cast<const T*>(a.k), static_cast<const T*>(a.v), a.s, a.log_decay,
                       a.from, a.parent, a.to, static_cast<T*>(a.o), Divisor(a.H), a.n_from, a.eps,
                       int(streamed(units, DK, DV)));
}
template <typename T, int DK, int DV, int COLS>
hipError_t accept_parts(const TreeArgs& a) {
  const int units = a.B * a.H;
  return launch_kernel("tree_accept_kernel", tree_accept_kernel<T, DK, DV, COLS>, dim3(units * (DV / COLS)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.k), static_cast<const T*>(a.v), a.log_decay, a.parent, a.last, a.state,
                       Divisor(a.H), a.n_tokens, a.eps, int(streamed(units, DK, DV)));
}

#define COTTN_STATE_SHAPES(CASE)                                                                                  \
  switch (a.dk * 1000 + a.dv) {                                                                                   \
    CASE(32, 32) CASE(32, 64) CASE(32, 128) CASE(64, 32) CASE(64, 64) CASE(64, 128) CASE(128, 32) CASE(128, 64)   \
    CASE(128, 128)                                                                                                \
    default: return hipErrorInvalidValue;                                                                         \
  }

template <typename T>
hipError_t run_step_decay(const StepDecayArgs& a) {
#define COTTN_CASE(DK, DV) \
  case DK * 1000 + DV: return state_parts(a.B * a.H, DV) ? step_parts<T, DK, DV, 32>(a) : step_parts<T, DK, DV, DV>(a);
  COTTN_STATE_SHAPES(COTTN_CASE)
#undef COTTN_CASE
}
template <typename T>
hipError_t run_tree_accept(const TreeArgs& a) {
#define COTTN_CASE(DK, DV) \
  case DK * 1000 + DV: return state_parts(a.B * a.H, DV) ? accept_parts<T, DK, DV, 32>(a) : accept_parts<T, DK, DV, DV>(a);
  COTTN_STATE_SHAPES(COTTN_CASE)
#undef COTTN_CASE
}

}  // namespace

hipError_t step_decay_any(const StepDecayArgs& a, int dtype) {
  return dtype == 0 ? run_step_decay<float>(a) : dtype == 1 ? run_step_decay<__bf16>(a) : run_step_decay<_Float16>(a);
}
hipError_t tree_accept_any(const TreeArgs& a, int dtype) {
  return dtype == 0 ? run_tree_accept<float>(a) : dtype == 1 ? run_tree_accept<__bf16>(a) : run_tree_accept<_Float16>(a);
}

}  // namespace cottn
