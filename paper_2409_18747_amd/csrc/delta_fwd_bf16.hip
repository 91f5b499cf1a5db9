// The gated delta rule, forward scan (formulas, precision: delta.h).
//
// A workgroup walks a (batch, head) chunk by chunk with VC of its value columns: those do not meet one another, the matrices W
// and P are the same for all.  The state is held in fp32 accumulators, and as parts in LDS, values down, for the products that
// read it.  A step is three products that wait for one another, Kh H, W (b Y) and Kh^T U, a barrier after each.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

template <typename T, int DK, int VC, int LEVEL>
struct DeltaFwdCfg {
  static constexpr int IN = Rows<T>::PARTS, OUT = RESULT_LEVEL<T>;
  using KTile = PartTile<CHUNK, DK, IN>;
  using State = PartTile<VC, DK, LEVEL>;     // [value][key]
  using Errors = PartTile<VC, CHUNK, LEVEL>; // [value][token]
  using Updates = PartTile<VC, CHUNK, OUT>;
  static constexpr int LDS_BYTES = 2 * (KTile::SIZE + State::SIZE + 2 * Errors::SIZE + Updates::SIZE) + CHUNK * 16;
  static constexpr int GROUPS = (160 * 1024) / LDS_BYTES >= 3 ? 3 : (160 * 1024) / LDS_BYTES >= 2 ? 2 : 1;
};

template <typename T, int DK, int VC, int LEVEL>
__global__ __launch_bounds__(256, (DeltaFwdCfg<T, DK, VC, LEVEL>::GROUPS)) void delta_fwd_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const float* __restrict__ s,
    const float* __restrict__ beta, const int* __restrict__ lengths, const float* state_in, T* __restrict__ O,
    float* state_out, const float* __restrict__ W, const double* __restrict__ decays,
    const float* __restrict__ factors, float* __restrict__ errors, float* __restrict__ states, Divisor H, Divisor parts, int N,
    int units, int DV, float eps) {
  using Cfg = DeltaFwdCfg<T, DK, VC, LEVEL>;
  using KTile = typename Cfg::KTile;
  using State = typename Cfg::State;
  using Errors = typename Cfg::Errors;
  using Updates = typename Cfg::Updates;
  using ST = StateTiles<DK, VC>;
  constexpr int IN = Cfg::IN, OUT = Cfg::OUT, KS = DK / 32, NT = VC / 16;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ss[State::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ys[Errors::SIZE];    // b Y
  __shared__ __attribute__((aligned(16))) uint16_t Us[Updates::SIZE];   // U
  __shared__ __attribute__((aligned(16))) uint16_t Ts[Errors::SIZE];    // U as it reaches the chunk's end
  __shared__ __attribute__((aligned(16))) double Gs[CHUNK];
  __shared__ __attribute__((aligned(16))) float rk[CHUNK], bs[CHUNK];
  fetch_argument_now(Q, K, V, s, beta, lengths, state_in, O, state_out, W, decays, factors, errors, states, H, parts, N, units,
                     DV, eps);
  int unit, part;
  unit_and_segment(blockIdx.x, units, parts, unit, part);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int there = valid_rows(lengths, unit, H, N), chunks = delta_chunks(N), steps = delta_chunks(there), col0 = part * VC;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* Vu = V + size_t(unit) * N * DV + col0;
  T* Ou = O + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  const int own = 16 * w + r;   // the token of the chunk whose row of Q, and of W, this lane holds pieces of

  f32x4 S[ST::NR][ST::NC];
#pragma unroll
  for (int x = 0; x < ST::NR; ++x)
#pragma unroll
    for (int y = 0; y < ST::NC; ++y) {
      S[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (state_in != nullptr && ST::active(w)) {
        const float* from = state_in + size_t(unit) * DK * DV + size_t(16 * ST::row_tile(w, x) + 4 * q4) * DV + col0 + 16 * ST::col_tile(w, y) + r;
#pragma unroll
        for (int v = 0; v < 4; ++v) S[x][y][v] = from[v * DV];
      }
    }

  RowTile<T, DK> kt;
  Raw8<T> qraw[KS];
  T vraw[NT][4];
  f32x4 wraw[2][2];
  double g_next = 0.0;
  float rk_next = 0.f, b_next = 0.f;
  const auto fetch_rows = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku, row0, there);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qraw[ks].zero();
      if (row0 + own < there) qraw[ks].load(Qu + size_t(row0 + own) * DK + 32 * ks + 8 * q4);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int row = row0 + 16 * w + 4 * q4 + v;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        vraw[t][v] = T(0.f);
        if (row < there) vraw[t][v] = Vu[size_t(row) * DV + 16 * t + r];
      }
    }
    if (tid < CHUNK) {
      const size_t at = (size_t(unit) * chunks + c) * CHUNK + tid;
      g_next = decays[at];
      rk_next = factors[at];
      b_next = row0 + tid < there ? beta[size_t(unit) * N + row0 + tid] : 0.f;
    }
  };
  const auto fetch_W = [&](int c) {
    const float* from = W + (size_t(unit) * chunks + c) * CHUNK * CHUNK + own * CHUNK + 8 * q4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (2 * ks <= w) wraw[ks][i] = *reinterpret_cast<const f32x4*>(from + 32 * ks + 4 * i);
  };
  if (steps > 0) {
    fetch_rows(0);
    fetch_W(0);
  }
  for (int c = 0; c < steps; ++c) {
    const int row0 = c * CHUNK;
    if (ST::active(w)) {
#pragma unroll
      for (int x = 0; x < ST::NR; ++x)
#pragma unroll
        for (int y = 0; y < ST::NC; ++y)
          State::store4(Ss, 16 * ST::col_tile(w, y) + r, 16 * ST::row_tile(w, x) + 4 * q4, S[x][y]);
    }
    if (states != nullptr && ST::active(w)) {
      float* to = states + (size_t(unit) * chunks + c) * DK * DV + col0;
#pragma unroll
      for (int x = 0; x < ST::NR; ++x)
#pragma unroll
        for (int y = 0; y < ST::NC; ++y)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            to[size_t(16 * ST::row_tile(w, x) + 4 * q4 + v) * DV + 16 * ST::col_tile(w, y) + r] = S[x][y][v];
    }
    kt.commit(Ks);
    if (tid < CHUNK) {
      Gs[tid] = g_next;
      rk[tid] = rk_next;
      bs[tid] = b_next;
    }
    __syncthreads();

    // what the state before the chunk gives: Kh H, tokens down, and Qh H, values down; and P, keys down
    f32x4 y[NT], o[NT];
    bf16x8 pf[2][OUT];
    {
      bf16x8 qf[KS][IN];
      float rq = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qraw[ks].parts(qf[ks]);
        rq += qraw[ks].sum_sq();
      }
      rq += __shfl_xor(rq, 16, 64);
      rq = inv_norm(rq + __shfl_xor(rq, 32, 64), eps);
#pragma unroll
      for (int t = 0; t < NT; ++t) y[t] = o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[IN], sf[NT][LEVEL];
        KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf);
#pragma unroll
        for (int t = 0; t < NT; ++t) State::row_frag(Ss, 16 * t + r, 32 * ks + 8 * q4, sf[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t) y[t] = mm<LEVEL>(kf, sf[t], y[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = mm<OUT>(sf[t], qf[ks], o[t]);
      }
      const double g_own = Gs[own];
      const float since = rq * decay_between(g_own, 0.0);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) o[t][v] *= since;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 half[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int jt = 2 * p + h;
          if (jt <= w) {
            f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              bf16x8 kf[IN];
              KTile::row_frag(Ks, 16 * jt + r, 32 * ks + 8 * q4, kf);
              t = mm<OUT>(kf, qf[ks], t);
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int j = 16 * jt + 4 * q4 + v;
              half[h][v] = j <= own ? t[v] * rk[j] * (rq * decay_between(g_own, Gs[j])) : 0.f;
            }
          }
        }
        split8<OUT>(half[0], half[1], pf[p]);
      }
    }
    float to_end[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = 16 * w + 4 * q4 + v;
      const float f = rk[i] * decay_between(Gs[i], 0.0);
      to_end[v] = rk[i] * decay_between(Gs[CHUNK - 1], Gs[i]);
#pragma unroll
      for (int t = 0; t < NT; ++t) y[t][v] = __builtin_fmaf(-f, y[t][v], float(vraw[t][v]));
    }
    const f32x4 b4 = *reinterpret_cast<const f32x4*>(bs + 16 * w + 4 * q4);
#pragma unroll
    for (int t = 0; t < NT; ++t) Errors::store4(Ys, 16 * t + r, 16 * w + 4 * q4, b4 * y[t]);
    const StateFactor kept(Gs[CHUNK - 1]);
    if (c + 1 < steps) fetch_rows(c + 1);
    __syncthreads();

    // the errors and the updates
    {
      f32x4 e[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) e[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        if (2 * ks <= w) {
          bf16x8 wf[LEVEL];
          split8<LEVEL>(wraw[ks][0], wraw[ks][1], wf);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8 yf[LEVEL];
            Errors::row_frag(Ys, 16 * t + r, 32 * ks + 8 * q4, yf);
            e[t] = mm<LEVEL>(wf, yf, e[t]);
          }
        }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        e[t] = y[t] - e[t];
        const f32x4 u = b4 * e[t];
        Updates::store4(Us, 16 * t + r, 16 * w + 4 * q4, u);
        Errors::store4(Ts, 16 * t + r, 16 * w + 4 * q4, f32x4{u[0] * to_end[0], u[1] * to_end[1], u[2] * to_end[2], u[3] * to_end[3]});
        if (errors != nullptr) {
          float* to = errors + ((size_t(unit) * chunks + c) * CHUNK + 16 * w + 4 * q4) * DV + col0 + 16 * t + r;
#pragma unroll
          for (int v = 0; v < 4; ++v) to[v * DV] = e[t][v];
        }
      }
      if (c + 1 < steps) fetch_W(c + 1);
    }
    __syncthreads();

    // the state behind the chunk, and the rows' results
    if (ST::active(w)) {
#pragma unroll
      for (int x = 0; x < ST::NR; ++x)
#pragma unroll
        for (int y_ = 0; y_ < ST::NC; ++y_)
#pragma unroll
          for (int v = 0; v < 4; ++v) S[x][y_][v] = kept.of(S[x][y_][v]);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        bf16x8 uf[ST::NC][LEVEL];
#pragma unroll
        for (int y_ = 0; y_ < ST::NC; ++y_) Errors::row_frag(Ts, 16 * ST::col_tile(w, y_) + r, 32 * ks + 8 * q4, uf[y_]);
#pragma unroll
        for (int x = 0; x < ST::NR; ++x) {
          bf16x8 kf[IN];
          KTile::col_frag(Ks, 32 * ks + 8 * q4, 32 * ks + 8 * q4 + 4, 16 * ST::row_tile(w, x), r, kf);
#pragma unroll
          for (int y_ = 0; y_ < ST::NC; ++y_) S[x][y_] = mm<LEVEL>(kf, uf[y_], S[x][y_]);
        }
      }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (2 * p <= w) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf16x8 uf[OUT];
          Updates::row_frag_pairs(Us, 16 * t + r, 32 * p + 4 * q4, uf);
          o[t] = mm<OUT>(uf, pf[p], o[t]);
        }
      }
    if (O != nullptr && row0 + own < there) {
      T* to = Ou + size_t(row0 + own) * DV + 4 * q4;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        typedef __attribute__((ext_vector_type(4))) T vec4;
        *reinterpret_cast<vec4*>(to + 16 * t) = vec4{T(scale * o[t][0]), T(scale * o[t][1]), T(scale * o[t][2]), T(scale * o[t][3])};
      }
    }
    __syncthreads();   // everything of the chunk is read
  }
  if (state_out != nullptr && ST::active(w)) {
    float* to = state_out + size_t(unit) * DK * DV + col0;
#pragma unroll
    for (int x = 0; x < ST::NR; ++x)
#pragma unroll
      for (int y = 0; y < ST::NC; ++y)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          to[size_t(16 * ST::row_tile(w, x) + 4 * q4 + v) * DV + 16 * ST::col_tile(w, y) + r] = S[x][y][v];
  }
  // rows that do not exist
  if (O == nullptr) return;
  for (long i = tid; i < long(N - there) * (VC / 4); i += 256) {
    typedef __attribute__((ext_vector_type(4))) T vec4;
    *reinterpret_cast<vec4*>(Ou + size_t(there + i / (VC / 4)) * DV + i % (VC / 4) * 4) = vec4{T(0.f), T(0.f), T(0.f), T(0.f)};
  }
}

template <typename T, int DK, int VC, int LEVEL>
hipError_t run_scan(const DeltaArgs& a) {
  const int units = a.B * a.H, parts = a.dv / VC;
  return launch_kernel("delta_fwd_scan", delta_fwd_scan<T, DK, VC, LEVEL>, dim3(unsigned(units * parts)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.V), a.s, a.beta, a.seq_len,
                       a.state_in, static_cast<T*>(a.O), a.state, a.W, a.decays, a.factors, a.errors, a.states, Divisor(a.H),
                       Divisor(parts), a.N, units, a.dv, a.eps);
}

template <typename T, int DK>
hipError_t run_shape(const DeltaArgs& a) {
  constexpr int MOST = 3;
  // without fp32 results two parts do
  if (sizeof(T) == 2 && a.state == nullptr && a.errors == nullptr) return run_scan<T, DK, 32, RESULT_LEVEL<T>>(a);
  return run_scan<T, DK, 32, MOST>(a);
}

}  // namespace

// (O null: for a backward, errors and states alone)
hipError_t DELTA_SYM(delta_fwd)(const DeltaArgs& a) {
  typedef DELTA_T T;
  const hipError_t err = DELTA_SYM(delta_prepare)(a);
  if (err != hipSuccess) return err;
  return a.dk == 32 ? run_shape<T, 32>(a) : a.dk == 64 ? run_shape<T, 64>(a) : run_shape<T, 128>(a);
}

}  // namespace cottn
