// One token by the gated delta rule for B H independent states, fp32 on the vector ALU:
//     w = beta (v - kh g S),   S <- g S + kh^T w,   o = s qh S = s (qh g S + (qh . kh) w).
// The state goes through the chip once: a workgroup owns COLS value columns of one, a row covered by COLS / 4 lanes, holds them
// all in registers and forms both column sums, over kh and over qh, in one pass before it writes the rows back.  What bounds it is
// HBM: 256 x 16 states of 128 x 128 in 108 us, 5.0 TB/s (80 us where the same states come again and again).
#include "device_common.h"
#include "launch.h"
#include "delta.h"

namespace cottn {
namespace {

template <int DK, int COLS>
struct StepRows {
  static constexpr int TPR = COLS / 4, RPP = 256 / TPR, PASSES = (DK + RPP - 1) / RPP;
  static constexpr bool WHOLE = DK % RPP == 0;
};

// parent == null: from the sequence's own place in `from`; else from that of sequence parent[b], from nothing where that is none
// of its n_from.
template <typename T, int DK, int COLS>
__global__ __launch_bounds__(256) void step_delta_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ s,
    const float* __restrict__ log_decay, const float* __restrict__ beta, const float* from, const int* __restrict__ parent,
    float* to, T* __restrict__ o, Divisor H, Divisor parts, int n_from, int DV, float eps, int stream) {
  using R = StepRows<DK, COLS>;
  __shared__ __attribute__((aligned(16))) float qh[DK], kh[DK];
  __shared__ __attribute__((aligned(16))) f32x4 sums[2][4][R::TPR];
  fetch_argument_now(q, k, v, s, log_decay, beta, from, parent, to, o, H, parts, n_from, DV, eps, stream);
  const int unit = quotient(blockIdx.x, parts), part = blockIdx.x - unit * parts.n, b = quotient(unit, H), head = unit - b * H.n;
  const int tid = threadIdx.x, w = tid / 64, l = tid % 64, lane = tid % R::TPR;
  const int col = part * COLS + 4 * lane, row0 = tid / R::TPR;
  int src = b;
  if (parent != nullptr) src = parent[b];
  const bool none = src < 0 || src >= n_from;
  const float* S = from + (size_t(none ? 0 : src) * H.n + head) * DK * DV;
  f32x4 rows[R::PASSES];
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    rows[p] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!none && (R::WHOLE || row < DK)) {
      const f32x4* at = reinterpret_cast<const f32x4*>(S + size_t(row) * DV + col);
      rows[p] = stream ? __builtin_nontemporal_load(at) : *at;
    }
  }
  float q0 = 0.f, q1 = 0.f, k0 = 0.f, k1 = 0.f;   // every wave: elements l and l + 64
  if (l < DK) {
    q0 = float(q[size_t(unit) * DK + l]);
    k0 = float(k[size_t(unit) * DK + l]);
  }
  if (DK > 64) {
    q1 = float(q[size_t(unit) * DK + 64 + l]);
    k1 = float(k[size_t(unit) * DK + 64 + l]);
  }
  typedef __attribute__((ext_vector_type(4))) T vec4;
  const vec4 vt = *reinterpret_cast<const vec4*>(v + size_t(unit) * DV + col);
  const float scale = s[head], b1 = beta[unit];
  float times, plus;
  state_factor(log_decay != nullptr ? log2_decay(log_decay[unit]) : 0.0, times, plus);
  // (bounded for zero rows, whose 1 / eps may be infinite: delta.h)
  const float rq = fminf(inv_norm(group_sum<64>(__builtin_fmaf(q0, q0, q1 * q1)), eps), LARGEST_FACTOR);
  const float rk = fminf(inv_norm(group_sum<64>(__builtin_fmaf(k0, k0, k1 * k1)), eps), LARGEST_FACTOR);
  q0 *= rq; q1 *= rq; k0 *= rk; k1 *= rk;
  const float qk = group_sum<64>(__builtin_fmaf(q0, k0, q1 * k1));
  if (w == 0) {
    if (l < DK) {
      qh[l] = q0;
      kh[l] = k0;
    }
    if (DK > 64) {
      qh[64 + l] = q1;
      kh[64 + l] = k1;
    }
  }
  __syncthreads();
  f32x4 by_k = {0.f, 0.f, 0.f, 0.f}, by_q = by_k;
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    if (R::WHOLE || row < DK) {
      const float kr = kh[row], qr = qh[row];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        rows[p][i] = __builtin_fmaf(rows[p][i], plus, rows[p][i] * times);
        by_k[i] = __builtin_fmaf(kr, rows[p][i], by_k[i]);
        by_q[i] = __builtin_fmaf(qr, rows[p][i], by_q[i]);
      }
    }
  }
  // over the rows that lanes of a wave hold, then over the waves
#pragma unroll
  for (int d = R::TPR; d < 64; d *= 2)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      by_k[i] += __shfl_xor(by_k[i], d, 64);
      by_q[i] += __shfl_xor(by_q[i], d, 64);
    }
  if (l < R::TPR) {
    sums[0][w][lane] = by_k;
    sums[1][w][lane] = by_q;
  }
  __syncthreads();
  by_k = (sums[0][0][lane] + sums[0][1][lane]) + (sums[0][2][lane] + sums[0][3][lane]);
  const f32x4 u = b1 * (f32x4{float(vt[0]), float(vt[1]), float(vt[2]), float(vt[3])} - by_k);
  float* out = to + size_t(unit) * DK * DV;
#pragma unroll
  for (int p = 0; p < R::PASSES; ++p) {
    const int row = p * R::RPP + row0;
    if (R::WHOLE || row < DK) {
      const float kr = kh[row];
      f32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(kr, u[i], rows[p][i]);
      __builtin_nontemporal_store(x, reinterpret_cast<f32x4*>(out + size_t(row) * DV + col));
    }
  }
  if (tid < R::TPR) {
    by_q = (sums[1][0][lane] + sums[1][1][lane]) + (sums[1][2][lane] + sums[1][3][lane]);
    vec4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = static_cast<T>(scale * __builtin_fmaf(qk, u[i], by_q[i]));
    *reinterpret_cast<vec4*>(o + size_t(unit) * DV + col) = y;
  }
}

template <typename T, int DK, int COLS>
hipError_t run_step(const StepDeltaArgs& a) {
  const StepDecayArgs& t = a.step;
  const int units = t.B * t.H, parts = t.dv / COLS;
  // non-temporal loads where the states of a call exceed the L2s, as in the other steps (512 of 128 x 128: 9.4 -> 8.6 us)
  const int stream = double(units) * t.dk * t.dv * sizeof(float) > 32.0 * 1024 * 1024;
  return launch_kernel("step_delta_kernel", step_delta_kernel<T, DK, COLS>, dim3(unsigned(units * parts)), dim3(256), 0, t.stream,
                       static_cast<const T*>(t.q), static_cast<const T*>(t.k), static_cast<const T*>(t.v), t.s, t.log_decay,
                       a.beta, t.from, t.parent, t.to, static_cast<T*>(t.o), Divisor(t.H), Divisor(parts), t.n_from, t.dv, t.eps,
                       stream);
}
template <typename T, int DK>
hipError_t run_width(const StepDeltaArgs& a) {
  // a state to several workgroups where there are few: 16 of 128 x 128 5.0 -> 4.6 us, 128 5.9 -> 5.5, 256 the same
  if (a.step.dv == 32 || a.step.B * a.step.H <= 128) return run_step<T, DK, 32>(a);
  return a.step.dv == 64 ? run_step<T, DK, 64>(a) : run_step<T, DK, 128>(a);
}
template <typename T>
hipError_t run_type(const StepDeltaArgs& a) {
  return a.step.dk == 32 ? run_width<T, 32>(a) : a.step.dk == 64 ? run_width<T, 64>(a) : run_width<T, 128>(a);
}

}  // namespace

hipError_t step_delta_any(const StepDeltaArgs& a, int dtype) {
  return dtype == 0 ? run_type<float>(a) : dtype == 1 ? run_type<__bf16>(a) : run_type<_Float16>(a);
}

}  // namespace cottn
