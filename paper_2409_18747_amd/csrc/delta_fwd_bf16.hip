// The gated delta rule, forward scan (formulas, precision: delta.h).
//
// A workgroup walks a (batch, head) chunk by chunk with VC of its value columns: those do not meet one another, the matrices W
// and P are the same for all.  The state is held in fp32 accumulators, values down, and as parts in LDS for the products that
// read it.  A step is three products that wait for one another, Kh H, W b Y and Kh^T U, a barrier after each.  Results lie
// transposed in the accumulators: a lane has four consecutive value columns of one token, whose factors it holds.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

template <typename T, int DK, int VC, int LEVEL>
struct DeltaFwdCfg {
  static constexpr int IN = Rows<T>::PARTS, OUT = RESULT_LEVEL<T>;
  using KTile = PartTile<CHUNK, DK, IN>;
  using State = PartTile<DK, VC, LEVEL>;      // [key][value]
  using Errors = PartTile<CHUNK, VC, LEVEL>;  // [token][value]
  using Updates = PartTile<CHUNK, VC, OUT>;
  // the state before the chunk, and when it is read the updates
  static constexpr int ROOM = State::SIZE > Errors::SIZE + Updates::SIZE ? State::SIZE : Errors::SIZE + Updates::SIZE;
  static constexpr int LDS_BYTES = 2 * (KTile::SIZE + ROOM + Errors::SIZE) + int(sizeof(ChunkRecord));
  static constexpr int GROUPS = (160 * 1024) / LDS_BYTES >= 3 ? 3 : (160 * 1024) / LDS_BYTES >= 2 ? 2 : 1;
};

template <typename T, int DK, int VC, int LEVEL>
__global__ __launch_bounds__(256, (DeltaFwdCfg<T, DK, VC, LEVEL>::GROUPS)) void delta_fwd_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* state_in, T* __restrict__ O, float* state_out,
    const ChunkRecord* __restrict__ records, const uint16_t* __restrict__ w_rows, float* __restrict__ errors,
    float* __restrict__ states, Divisor H, Divisor parts, int N, int units, int DV, float inv_eps) {
  using Cfg = DeltaFwdCfg<T, DK, VC, LEVEL>;
  using KTile = typename Cfg::KTile;
  using State = typename Cfg::State;
  using Errors = typename Cfg::Errors;
  using Updates = typename Cfg::Updates;
  using ST = StateTiles<DK, VC>;
  constexpr int IN = Cfg::IN, OUT = Cfg::OUT, KS = DK / 32, NT = VC / 16;
  typedef __attribute__((ext_vector_type(4))) T vec4;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t room[Cfg::ROOM];
  __shared__ __attribute__((aligned(16))) uint16_t Ys[Errors::SIZE];
  __shared__ ChunkRecord rec;
  uint16_t* const Ss = room;
  uint16_t* const Ts = room;                  // U as it reaches the chunk's end
  uint16_t* const Us = room + Errors::SIZE;   // U
  fetch_argument_now(Q, K, V, s, lengths, state_in, O, state_out, records, w_rows, errors, states, H, parts, N, units, DV, inv_eps);
  int unit, part;
  unit_and_segment(blockIdx.x, units, parts, unit, part);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int there = valid_rows(lengths, unit, H, N), chunks = delta_chunks(N), steps = delta_chunks(there), col0 = part * VC;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* Vu = V + size_t(unit) * N * DV + col0;
  T* Ou = O + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  const int own = 16 * w + r;   // this lane's token of the chunk
  const unsigned own_q = unsigned(own * DK + 8 * q4), own_v = unsigned(own * DV + 4 * q4);
  const bool active = ST::active(w);

  const auto state_at = [&](int x, int y) {
    return unsigned((16 * ST::key_tile(w, y) + r) * DV + col0 + 16 * ST::value_tile(w, x) + 4 * q4);
  };
  f32x4 S[ST::NV][ST::NK];
#pragma unroll
  for (int x = 0; x < ST::NV; ++x)
#pragma unroll
    for (int y = 0; y < ST::NK; ++y) {
      S[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (state_in != nullptr && active) S[x][y] = *reinterpret_cast<const f32x4*>(state_in + size_t(unit) * DK * DV + state_at(x, y));
    }

  RowTile<T, DK> kt;
  Raw8<T> qraw[KS];
  vec4 vraw[NT];
  u32x4 rec_next = {0u, 0u, 0u, 0u};
  bf16x8 wf[2][LEVEL];
  const auto fetch_rows = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku + size_t(row0) * DK, there - row0);
    const T* Qc = Qu + size_t(row0) * DK;
    const T* Vc = Vu + size_t(row0) * DV;
    if (row0 + own < there) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qraw[ks].load(Qc + own_q + 32 * ks);
#pragma unroll
      for (int t = 0; t < NT; ++t) vraw[t] = *reinterpret_cast<const vec4*>(Vc + own_v + 16 * t);
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qraw[ks].zero();
#pragma unroll
      for (int t = 0; t < NT; ++t) vraw[t] = vec4{T(0.f), T(0.f), T(0.f), T(0.f)};
    }
    if (tid < RECORD_PIECES) rec_next = reinterpret_cast<const u32x4*>(records + size_t(unit) * chunks + c)[tid];
  };
  const auto fetch_W = [&](int c) {
    const uint16_t* from = w_rows + (size_t(unit) * chunks + c) * W_ELEMS;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < LEVEL; ++i)
        if (w_row_there(w, ks))
          wf[ks][i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(from + w_row_frag(w, ks) * 3 * 512 + i * 512 + l * 8));
  };
  if (steps > 0) {
    fetch_rows(0);
    fetch_W(0);
  }
  for (int c = 0; c < steps; ++c) {
    const int row0 = c * CHUNK;
    if (active) {
#pragma unroll
      for (int x = 0; x < ST::NV; ++x)
#pragma unroll
        for (int y = 0; y < ST::NK; ++y)
          State::store4(Ss, 16 * ST::key_tile(w, y) + r, 16 * ST::value_tile(w, x) + 4 * q4, S[x][y]);
      if (states != nullptr) {
        float* to = states + (size_t(unit) * chunks + c) * DK * DV;
#pragma unroll
        for (int x = 0; x < ST::NV; ++x)
#pragma unroll
          for (int y = 0; y < ST::NK; ++y) *reinterpret_cast<f32x4*>(to + state_at(x, y)) = S[x][y];
      }
    }
    kt.commit(Ks);
    if (tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[tid] = rec_next;
    __syncthreads();

    // what the state before the chunk gives: Kh H and Qh H; and P, keys down
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
      rq = row_factor(rq + __shfl_xor(rq, 32, 64), inv_eps);
#pragma unroll
      for (int t = 0; t < NT; ++t) y[t] = o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[IN], sf[NT][LEVEL];
        KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf);
#pragma unroll
        for (int t = 0; t < NT; ++t) State::col_frag(Ss, 32 * ks + 8 * q4, 32 * ks + 8 * q4 + 4, 16 * t, r, sf[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t) y[t] = mm<LEVEL>(sf[t], kf, y[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = mm<OUT>(sf[t], qf[ks], o[t]);
      }
      const float before = -rec.rk_since[own];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int v = 0; v < 4; ++v) y[t][v] = __builtin_fmaf(before, y[t][v], float(vraw[t][v]));
        Errors::store4(Ys, own, 16 * t + 4 * q4, y[t]);
      }
      const float since = rq * rec.since[own];
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= since;
      const float in_tile = rq * rec.in_tile[own];
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
            if (jt < w) {
              half[h] = t * *reinterpret_cast<const f32x4*>(rec.rk_to_tile + 16 * jt + 4 * q4) * (in_tile * rec.between[w][jt]);
            } else {
              const double g_own = rec.decay[own];
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const int j = 16 * jt + 4 * q4 + v;
                half[h][v] = j <= own ? t[v] * rec.rk[j] * (rq * decay_between(g_own, rec.decay[j])) : 0.f;
              }
            }
          }
        }
        split8<OUT>(half[0], half[1], pf[p]);
      }
    }
    const float b = rec.beta[own], b_to_end = b * rec.rk_to_end[own], times = rec.times, plus = rec.plus;
    if (c + 1 < steps) fetch_rows(c + 1);
    __syncthreads();

    // the errors and the updates
    {
      f32x4 e[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) e[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        if (w_row_there(w, ks)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8 yf[LEVEL];
            Errors::col_frag(Ys, 32 * ks + 8 * q4, 32 * ks + 8 * q4 + 4, 16 * t, r, yf);
            e[t] = mm<LEVEL>(yf, wf[ks], e[t]);
          }
        }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        e[t] = y[t] - e[t];
        Errors::store4(Ts, own, 16 * t + 4 * q4, b_to_end * e[t]);
        Updates::store4(Us, own, 16 * t + 4 * q4, b * e[t]);
      }
      if (errors != nullptr) {
        float* to = errors + (size_t(unit) * chunks + c) * CHUNK * DV + col0 + own_v;
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(to + 16 * t) = e[t];
      }
      if (c + 1 < steps) fetch_W(c + 1);
    }
    __syncthreads();

    // the state behind the chunk, and the rows' results
    if (active) {
#pragma unroll
      for (int x = 0; x < ST::NV; ++x)
#pragma unroll
        for (int k = 0; k < ST::NK; ++k)
#pragma unroll
          for (int v = 0; v < 4; ++v) S[x][k][v] = __builtin_fmaf(S[x][k][v], plus, S[x][k][v] * times);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int t0 = 32 * ks + 8 * q4;
        bf16x8 uf[ST::NV][LEVEL];
#pragma unroll
        for (int x = 0; x < ST::NV; ++x) Errors::col_frag(Ts, t0, t0 + 4, 16 * ST::value_tile(w, x), r, uf[x]);
#pragma unroll
        for (int k = 0; k < ST::NK; ++k) {
          bf16x8 kf[IN];
          KTile::col_frag(Ks, t0, t0 + 4, 16 * ST::key_tile(w, k), r, kf);
#pragma unroll
          for (int x = 0; x < ST::NV; ++x) S[x][k] = mm<LEVEL>(uf[x], kf, S[x][k]);
        }
      }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (2 * p <= w) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf16x8 uf[OUT];
          Updates::col_frag(Us, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * t, r, uf);
          o[t] = mm<OUT>(uf, pf[p], o[t]);
        }
      }
    if (O != nullptr && row0 + own < there) {
      T* to = Ou + size_t(row0) * DV + own_v;
#pragma unroll
      for (int t = 0; t < NT; ++t)
        *reinterpret_cast<vec4*>(to + 16 * t) = vec4{T(scale * o[t][0]), T(scale * o[t][1]), T(scale * o[t][2]), T(scale * o[t][3])};
    }
    __syncthreads();   // everything of the chunk is read
  }
  if (state_out != nullptr && active) {
#pragma unroll
    for (int x = 0; x < ST::NV; ++x)
#pragma unroll
      for (int y = 0; y < ST::NK; ++y) *reinterpret_cast<f32x4*>(state_out + size_t(unit) * DK * DV + state_at(x, y)) = S[x][y];
  }
  // rows that do not exist
  if (O == nullptr) return;
  for (long i = tid; i < long(N - there) * (VC / 4); i += 256)
    *reinterpret_cast<vec4*>(Ou + size_t(there + i / (VC / 4)) * DV + i % (VC / 4) * 4) = vec4{T(0.f), T(0.f), T(0.f), T(0.f)};
}

template <typename T, int DK, int VC, int LEVEL>
hipError_t run_scan(const DeltaArgs& a) {
  const int units = a.B * a.H, parts = a.dv / VC;
  return launch_kernel("delta_fwd_scan", delta_fwd_scan<T, DK, VC, LEVEL>, dim3(unsigned(units * parts)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.V), a.s, a.seq_len,
                       a.state_in, static_cast<T*>(a.O), a.state, static_cast<const ChunkRecord*>(a.records), a.w_rows, a.errors,
                       a.states, Divisor(a.H), Divisor(parts), a.N, units, a.dv, 1.0f / a.eps);
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
