// Rotary positions with several axes.  Pair p of a row's features, (x_a, x_b), is turned by the angle
//     phi = position[b][n][axis[p]] freq[p]:   y_a = x_a cos phi - x_b sin phi,   y_b = x_b cos phi + x_a sin phi
// (inverse: by - phi, which is also the gradient).  Features of no pair are copied.
//
// Rows go through the chip once, which is what bounds it: 8 x 16 heads of 4608 rows of 128 in 121 us, 4.97 TB/s of reads and writes
// (a copy of 1 GiB: 5.17).  Sines and cosines are formed once for all heads of Q and K that a workgroup takes.  A position times a frequency is formed, and whole turns are taken off it, in 64 bits: in 32 an angle of
// position 10^6 would be off by 0.03.  What is left, at most half a turn, is a sine's argument in fp32.
#include "device_common.h"
#include "launch.h"

namespace cottn {
using namespace COTTN_NS;
namespace {

template <typename T, int N> struct alignas(N * sizeof(T)) Run { T x[N]; };

// A thread owns VEC pairs of one token: features a .. and b .. (halves), or 2 VEC features from a on (neighbours).  A workgroup
// takes 256 / LPT tokens, LPT lanes to a token, and the heads h0 .. h1 - 1 of both tensors.
template <typename T, int VEC, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(const T* Q, const T* K, const int* __restrict__ positions,
                                                     const float* __restrict__ freq, const int* __restrict__ axis, T* Qr, T* Kr,
                                                     int H, int N, int d, int pairs, int axes, float sign, int lanes, int tiles,
                                                     int heads_each) {
  const int per = 256 / lanes, b = blockIdx.x / tiles, tile = blockIdx.x - b * tiles;
  const int n = tile * per + int(threadIdx.x) / lanes, lane = int(threadIdx.x) % lanes;
  if (int(threadIdx.x) / lanes >= per || n >= N) return;
  const int h0 = blockIdx.y * heads_each, h1 = min(H, h0 + heads_each);
  const int turning = pairs / VEC;                  // lanes with pairs; the ones behind copy 2 VEC features each
  const bool turns = lane < turning;
  const int first = NEIGHBOURS || !turns ? 2 * VEC * lane : VEC * lane, second = NEIGHBOURS || !turns ? first + VEC : first + pairs;
  float c[VEC], s[VEC];
  bool turned[VEC];   // (a pair of an axis that there is not stays as it is, whatever its features are: no 0 times infinity)
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
    turned[i] = false;
    if (turns) {
      const int p = VEC * lane + i;
      const int ax = axis != nullptr ? axis[p] : 0;
      if (ax >= 0 && ax < axes) {
        const double turn = double(positions[(size_t(b) * N + n) * axes + ax]) * double(freq[p]) * 0.15915494309189535;
        float si, co;
        sincospif(2.f * float(turn - rint(turn)), &si, &co);
        c[i] = co;
        s[i] = sign * si;
        turned[i] = true;
      }
    }
  }
  const auto turn_rows = [&](const T* from, T* to) {
    const size_t step = size_t(N) * d;
    size_t at = (size_t(b) * H + h0) * step + size_t(n) * d;
    for (int h = h0; h < h1; ++h, at += step) {
      Run<T, VEC> x = *reinterpret_cast<const Run<T, VEC>*>(from + at + first);
      Run<T, VEC> y = *reinterpret_cast<const Run<T, VEC>*>(from + at + second);
      if (turns) {
        if constexpr (NEIGHBOURS) {
          T z[2 * VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            z[i] = x.x[i];
            z[VEC + i] = y.x[i];
          }
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float u = float(z[2 * i]), v = float(z[2 * i + 1]);
            z[2 * i] = turned[i] ? T(__builtin_fmaf(u, c[i], -(v * s[i]))) : z[2 * i];
            z[2 * i + 1] = turned[i] ? T(__builtin_fmaf(v, c[i], u * s[i])) : z[2 * i + 1];
          }
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            x.x[i] = z[i];
            y.x[i] = z[VEC + i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float u = float(x.x[i]), v = float(y.x[i]);
            x.x[i] = turned[i] ? T(__builtin_fmaf(u, c[i], -(v * s[i]))) : x.x[i];
            y.x[i] = turned[i] ? T(__builtin_fmaf(v, c[i], u * s[i])) : y.x[i];
          }
        }
      }
      *reinterpret_cast<Run<T, VEC>*>(to + at + first) = x;
      *reinterpret_cast<Run<T, VEC>*>(to + at + second) = y;
    }
  };
  turn_rows(Q, Qr);
  if (K != nullptr) turn_rows(K, Kr);
}

template <typename T, int VEC, bool NEIGHBOURS>
hipError_t run_rotary(const RotaryArgs& a) {
  const int lanes = a.d / (2 * VEC), tiles = int(rotary_tiles(a.N, a.d, VEC));
  // all heads to a workgroup where tokens alone fill the chip, else fewer (16 heads of one token: 4.5 us, of 1024 tokens 4.6; all to
  // a workgroup 15.6, 16.7)
  int heads = a.H;
  while (heads > 1 && long(a.B) * tiles * ((a.H + heads - 1) / heads) < 1024) heads = (heads + 1) / 2;
  return launch_kernel("rotary_kernel", rotary_kernel<T, VEC, NEIGHBOURS>, dim3(unsigned(a.B) * unsigned(tiles), unsigned((a.H + heads - 1) / heads)),
                       dim3(256), 0, a.stream, static_cast<const T*>(a.Q), static_cast<const T*>(a.K), a.positions, a.freq, a.axis,
                       static_cast<T*>(a.Qr), static_cast<T*>(a.Kr), a.H, a.N, a.d, a.pairs, a.axes, a.inverse ? -1.f : 1.f,
                       lanes, tiles, heads);
}
template <typename T>
hipError_t run_type(const RotaryArgs& a) {
  constexpr int VEC = 16 / sizeof(T);
  if (rotary_run(a.N, a.d, a.pairs, sizeof(T) == 4 ? 0 : 1) != VEC) return a.neighbours ? run_rotary<T, 1, true>(a) : run_rotary<T, 1, false>(a);
  return a.neighbours ? run_rotary<T, VEC, true>(a) : run_rotary<T, VEC, false>(a);
}

}  // namespace

hipError_t rotary_any(const RotaryArgs& a, int dtype) {
  return dtype == 0 ? run_type<float>(a) : dtype == 1 ? run_type<__bf16>(a) : run_type<_Float16>(a);
}

}  // namespace cottn
