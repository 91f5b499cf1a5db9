// The gated delta rule, segments of a sequence: the states at their starts, H_(g+1) = M_g H_g + B_g from the first on, or the
// gradients with respect to the states at their ends, D_(g-1) = M_g^T D_g + R_g from the last on, in place of B and R.
//
// A workgroup has 16 value columns and a wave 16 of the keys: a step is a row of M's tiles to each, and the state's parts go
// from all waves to all through the LDS.  What bounds it is the chain of segments, about 1.1 us a segment (16 heads of 64 x 64 in
// 16 of them: 17 us); M and B of the next one are on their way meanwhile.
#include "device_common.h"
#include "delta.h"

namespace cottn {
namespace {

template <int DK, bool REVERSE>
__global__ __launch_bounds__(4 * DK) void delta_carry(float* slots, const float* __restrict__ transitions,
                                                      const int* __restrict__ lengths, Divisor H, Divisor parts, int G, int seg, int N,
                                                      int DV) {
  constexpr int KS = DK / 32;
  __shared__ __attribute__((aligned(16))) uint16_t Xs[2][KS * 3 * 512];   // the state before a step, fragments of three parts
  const int unit = quotient(blockIdx.x, parts), part = blockIdx.x - unit * parts.n;
  const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 64), l = threadIdx.x % 64, r = l % 16, q4 = l / 16;
  const int all = delta_chunks(valid_rows(lengths, unit, H, N)), last = (all + seg - 1) / seg - 1;   // of the segments with rows
  // forward: from slot 1, segments 1 .. last - 1; reverse: from slot last - 1, segments last - 1 .. 1
  const int n = last - 1, start = REVERSE ? last - 1 : 1, step = REVERSE ? -1 : 1;
  if (n < 1) return;
  float* base = slots + size_t(unit) * G * DK * DV + key_of(w / 2, w % 2, 0, 0) * DV;
  const unsigned at_key = unsigned(8 * q4 * DV + 16 * part + r);
  const int key = key_of(w / 2, w % 2, r / 4, r % 4);   // the row of the product that this lane's row of the operand makes
  const auto load = [&](int slot) {
    f32x4 x;
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = (base + size_t(slot) * DK * DV + v * DV)[at_key];
    return x;
  };
  f32x4 m[KS][2], next;
  const auto fetch = [&](int g) {
    const float* M = transitions + (size_t(unit) * G + g) * DK * DK;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int from = 32 * ks + 8 * q4 + 4 * h;
        if (REVERSE) {
#pragma unroll
          for (int v = 0; v < 4; ++v) m[ks][h][v] = M[(from + v) * DK + key];
        } else {
          m[ks][h] = four(M + key * DK + from);
        }
      }
    next = load(g + step);
  };
  f32x4 x = load(start);
  fetch(start);
  for (int i = 0; i < n; ++i) {
    const int g = start + i * step;
    uint16_t* const X = Xs[i % 2];
    uint2 parts_[3];
    split4<3>(x, parts_);
#pragma unroll
    for (int p = 0; p < 3; ++p) reinterpret_cast<uint2*>(X)[((w / 2 * 3 + p) * 64 + l) * 2 + w % 2] = parts_[p];
    bf16x8 mf[KS][3];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) split8<3>(m[ks][0], m[ks][1], mf[ks]);
    x = next;
    if (i + 1 < n) fetch(g + step);
    lds_barrier();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 xf[3];
      load_frag(X, ks, l, xf);
      x = mm<3>(mf[ks], xf, x);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) (base + size_t(g + step) * DK * DV + v * DV)[at_key] = x[v];
  }
}

}  // namespace

hipError_t launch_delta_carry(const DeltaArgs& a, bool reverse) {
  const int units = a.B * a.H, parts = a.dv / 16;
  const auto run = [&](auto kernel) {
    return launch_kernel("delta_carry", kernel, dim3(unsigned(units * parts)), dim3(4 * a.dk), 0, a.stream, reverse ? a.ends : a.starts,
                         a.transitions, a.seq_len, Divisor(a.H), Divisor(parts), a.G, a.seg, a.N, a.dv);
  };
  if (reverse) return a.dk == 32 ? run(delta_carry<32, true>) : a.dk == 64 ? run(delta_carry<64, true>) : run(delta_carry<128, true>);
  return a.dk == 32 ? run(delta_carry<32, false>) : a.dk == 64 ? run(delta_carry<64, false>) : run(delta_carry<128, false>);
}

}  // namespace cottn
