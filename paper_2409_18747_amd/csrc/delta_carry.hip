// The gated delta rule, segments of a sequence: the states at their starts, H_(g+1) = M_g H_g + B_g from the first on, or the
// gradients with respect to the states at their ends, D_(g-1) = M_g^T D_g + R_g from the last on, in place of B and R.
//
// A wave has 16 value columns; the state goes on as the next product's operand in its accumulators, as in the scans (delta.h).
// What bounds it is the chain of segments: a step is M's way from the L2 and its taking apart.
#include "device_common.h"
#include "delta.h"

namespace cottn {
namespace {

template <int DK, bool REVERSE>
__global__ __launch_bounds__(128) void delta_carry(float* slots, const float* __restrict__ transitions,
                                                   const int* __restrict__ lengths, Divisor H, Divisor parts, int G, int seg, int N,
                                                   int DV) {
  constexpr int KS = DK / 32;
  const int unit = quotient(blockIdx.x, parts), part = blockIdx.x - unit * parts.n;
  const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 64), l = threadIdx.x % 64, r = l % 16, q4 = l / 16;
  const int all = delta_chunks(valid_rows(lengths, unit, H, N)), last = (all + seg - 1) / seg - 1;   // of the segments with rows
  const unsigned at_key = unsigned(8 * q4 * DV + 32 * part + 16 * w + r);
  float* base = slots + size_t(unit) * G * DK * DV;
  const auto load = [&](int slot, f32x4 (&x)[2 * KS]) {
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) x[t][v] = (base + size_t(slot) * DK * DV + key_of(t / 2, t % 2, 0, v) * DV)[at_key];
  };
  // forward: from slot 1, segments 1 .. last - 1; reverse: from slot last - 1, segments last - 1 .. 1
  const int n = last - 1;
  if (n < 1) return;
  f32x4 x[2 * KS];
  load(REVERSE ? last - 1 : 1, x);
  for (int i = 0; i < n; ++i) {
    const int g = REVERSE ? last - 1 - i : 1 + i, to = REVERSE ? g - 1 : g + 1;
    const float* M = transitions + (size_t(unit) * G + g) * DK * DK;
    f32x4 next[2 * KS];
    load(to, next);
    bf16x8 xf[KS][3];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) split8<3>(x[2 * ks], x[2 * ks + 1], xf[ks]);
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) {
      const int key = key_of(t / 2, t % 2, r / 4, r % 4);   // the row of the product that this lane's row of the operand makes
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        f32x4 lo, hi;
        if (REVERSE) {
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            lo[v] = M[(32 * ks + 8 * q4 + v) * DK + key];
            hi[v] = M[(32 * ks + 8 * q4 + 4 + v) * DK + key];
          }
        } else {
          lo = four(M + key * DK + 32 * ks + 8 * q4);
          hi = four(M + key * DK + 32 * ks + 8 * q4 + 4);
        }
        bf16x8 mf[3];
        split8<3>(lo, hi, mf);
        next[t] = mm<3>(mf, xf[ks], next[t]);
      }
    }
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) {
      x[t] = next[t];
#pragma unroll
      for (int v = 0; v < 4; ++v) (base + size_t(to) * DK * DV + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = x[t][v];
    }
  }
}

}  // namespace

hipError_t launch_delta_carry(const DeltaArgs& a, bool reverse) {
  const int units = a.B * a.H, parts = a.dv / 32;
  const auto run = [&](auto kernel) {
    return launch_kernel("delta_carry", kernel, dim3(unsigned(units * parts)), dim3(128), 0, a.stream, reverse ? a.ends : a.starts,
                         a.transitions, a.seq_len, Divisor(a.H), Divisor(parts), a.G, a.seg, a.N, a.dv);
  };
  if (reverse) return a.dk == 32 ? run(delta_carry<32, true>) : a.dk == 64 ? run(delta_carry<64, true>) : run(delta_carry<128, true>);
  return a.dk == 32 ? run(delta_carry<32, false>) : a.dk == 64 ? run(delta_carry<64, false>) : run(delta_carry<128, false>);
}

}  // namespace cottn
