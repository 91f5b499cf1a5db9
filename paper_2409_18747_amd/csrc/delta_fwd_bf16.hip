// The gated delta rule, forward scan (formulas, precision: delta.h).
//
// A workgroup walks a (batch, head) chunk by chunk, a wave for every 16 of its value columns: those do not meet one another, the
// rows of K and Q and the matrices W and P are the same for all.  A step is three products that wait for one another, Kh H, W b Y
// and Kh^T U.  Each is formed for the wave's columns with the tokens (or keys) down, and so is the next one's operand in the
// lanes that it is needed in: the state, Y and U never leave the wave's registers.
//   What nothing waits for is done beside that by twice as many waves more.  One half fetches the rows of the next chunk; the other
// forms P, and of the parts of the state and of U that the first waves leave in LDS the results, Q H + P U, transposed, so that
// four consecutive columns of a token are in a lane.
//   Prompts of 32 x 16 heads of 2048 rows at 128 x 128 take 564 us, with rows of tokens to a wave instead, and states and errors
// handed round through LDS, 811.  What bounds it: a step of some 8000 cycles (6000 at 64 x 64) in which the three kinds of waves,
// one of each to a SIMD, take turns: vector instructions issue in 52 % of the cycles, matrix instructions in 40, the LDS moves in
// 44; HBM gives 1.5 TB/s.  Neither W a chunk earlier in the LDS (so that the first waves never wait for it) nor splits into parts
// by one instruction less a value changed that by more than 3 %.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

template <typename T, int DK, int NW>
struct DeltaFwdCfg {
  static constexpr int LEVEL = 3, IN = Rows<T>::PARTS, OUT = RESULT_LEVEL<T>, VC = 16 * NW, KS = DK / 32;
  using KTile = PartTile<CHUNK, DK, IN>;
  using VTile = PartTile<CHUNK, VC, IN>;
  static constexpr int W_SIZE = W_FRAGS * LEVEL * 512, P_SIZE = W_FRAGS * OUT * 512, S_SIZE = NW * KS * OUT * 512, U_SIZE = NW * 2 * OUT * 512;
  static constexpr int BYTES = 2 * (2 * KTile::SIZE + W_SIZE + P_SIZE + S_SIZE + U_SIZE) + int(sizeof(ChunkRecord)) + 4 * CHUNK;
  // rows of V by way of the LDS (transposed on the way out), where it has room for them (32 x 16 heads of 1024 rows at 64 x 64
  // 125 us, by two bytes from memory 309; 512 rows at 128 x 128 142, 330)
  static constexpr bool V_IN_LDS = BYTES + 2 * VTile::SIZE <= 160 * 1024;
  static constexpr bool FITS = BYTES <= 160 * 1024;
};

// A sequence in G segments of `seg` chunks: the workgroups of TOTALS leave what a segment makes of a state, B from zeros (the first
// segment: from state_in) in the place of the state behind it, and the matrix M that the state at its start enters with, as if
// unit columns without values were its state; delta_carry makes of those the states at the starts, from which the segments are
// walked again.  Where the state is to replace state_in, which the last segment may do before the first one is walked again,
// the walk for the totals puts state_in by.
template <typename T, int DK, int NW, bool TOTALS>
__global__ __launch_bounds__((TOTALS ? 128 : 192) * NW, NW <= 2 ? 1 : TOTALS ? 2 : 3) void delta_fwd_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* state_in, T* __restrict__ O, float* state_out,
    const ChunkRecord* __restrict__ records, const uint16_t* __restrict__ w_rows, float* __restrict__ errors,
    float* __restrict__ states, float* starts, float* __restrict__ transitions, Divisor H, Divisor G, Divisor parts, int seg, int N,
    int units, int DV, float inv_eps) {
  using Cfg = DeltaFwdCfg<T, DK, NW>;
  using KTile = typename Cfg::KTile;
  using VTile = typename Cfg::VTile;
  constexpr int LEVEL = Cfg::LEVEL, IN = Cfg::IN, OUT = Cfg::OUT, KS = Cfg::KS, NT = 64 * NW, VC = Cfg::VC;
  typedef __attribute__((ext_vector_type(4))) T vec4;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[Cfg::V_IN_LDS ? VTile::SIZE : 8];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[Cfg::W_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[Cfg::P_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ss[Cfg::S_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Us[Cfg::U_SIZE];
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK];
  fetch_argument_now(Q, K, V, s, lengths, state_in, O, state_out, records, w_rows, errors, states, starts, transitions, H, G, parts, seg,
                     N, units, DV, inv_eps);
  int unit, part, g = 0;
  if (G.n == 1) {
    unit_and_segment(blockIdx.x, units, parts, unit, part);
  } else {   // (blockIdx.y: the part)
    unit_and_segment(blockIdx.x, units, G, unit, g);
    part = blockIdx.y;
  }
  const int tid = threadIdx.x % NT, role = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / NT);
  const int w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int there = valid_rows(lengths, unit, H, N), chunks = delta_chunks(N), all = delta_chunks(there), first = g * seg, steps = min(all, first + seg);
  const bool ends_here = steps == all && (first < all || g == 0);   // the state after the last row
  // TOTALS: columns of M, behind those of the values
  const bool unit_columns = TOTALS && part * VC >= DV;
  const int col0 = unit_columns ? part * VC - DV : part * VC, width = unit_columns ? DK : DV;
  const bool put_by = g == 0 && G.n > 1 && !ends_here && state_in != nullptr && state_in == state_out;
  if (TOTALS && (first >= all || (unit_columns ? g == 0 : ends_here))) return;   // (nobody asks)

  if (role == 0) {
    // ---- the states
    const T* Vu = V + size_t(unit) * N * DV + col0;
    // this lane's value column in the first key row, and in the first token row, that it holds
    const unsigned at_key = unsigned(8 * q4 * width + col0 + 16 * w + r), at_token = unsigned(4 * q4 * DV + col0 + 16 * w + r);
    f32x4 S[2 * KS];
    const float* from = g == 0 && (TOTALS || !put_by) ? (state_in != nullptr ? state_in + size_t(unit) * DK * DV : nullptr)
                        : TOTALS ? nullptr : starts + (size_t(unit) * G.n + g) * DK * DV;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        S[t][v] = from != nullptr ? (from + key_of(t / 2, t % 2, 0, v) * DV)[at_key] : 0.f;
        if (unit_columns) S[t][v] = key_of(t / 2, t % 2, q4, v) == col0 + 16 * w + r ? 1.f : 0.f;
      }
    if (TOTALS && put_by) {
      float* to = starts + size_t(unit) * G.n * DK * DV;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = S[t][v];
    }
    for (int c = first; c < steps; ++c) {
      bf16x8 sf[KS][LEVEL];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        split8<LEVEL>(S[2 * ks], S[2 * ks + 1], sf[ks]);
        if constexpr (!TOTALS) store_frag<OUT>(Ss, w * KS + ks, l, sf[ks]);
      }
      if (!TOTALS && states != nullptr) {
        float* to = states + (size_t(unit) * chunks + c) * DK * DV;
        const int ld = in_this_step(DV);
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * ld)[at_key] = S[t][v];
      }
      f32x4 y[4];
      if constexpr (!Cfg::V_IN_LDS) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int row = c * CHUNK + 16 * t + v;
            y[t][v] = !unit_columns && row + 4 * q4 < there ? float((Vu + size_t(row) * DV)[unsigned(4 * q4 * DV + 16 * w + r)]) : 0.f;
          }
      }
      lds_barrier();   // the chunk is there
      f32x4 kh[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) kh[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[4][IN];
#pragma unroll
        for (int t = 0; t < 4; ++t) KTile::row_frag(Ks, 16 * t + r, 32 * ks + 8 * q4, kf[t]);
        mm_each<LEVEL>(kf, sf[ks], kh);
      }
      bf16x8 yf[2][LEVEL];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (Cfg::V_IN_LDS) y[t] = unit_columns ? f32x4{0.f, 0.f, 0.f, 0.f} : VTile::col4(Vs, 16 * t + 4 * q4, 16 * w, r);
        const f32x4 since = four(rec.rk_since + 16 * t + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) y[t][v] = __builtin_fmaf(-since[v], kh[t][v], y[t][v]);
      }
      split8<LEVEL>(y[0], y[1], yf[0]);
      split8<LEVEL>(y[2], y[3], yf[1]);
      f32x4 e[4];
      {
        bf16x8 wf[4][LEVEL], wl[2][LEVEL];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          e[t] = f32x4{0.f, 0.f, 0.f, 0.f};
          load_frag(Ws, w_row_frag(t, 0), l, wf[t]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) load_frag(Ws, w_row_frag(2 + t, 1), l, wl[t]);
        mm_each<LEVEL>(wf, yf[0], e);
        mm_each<LEVEL>(wl, yf[1], e + 2);
      }
      bf16x8 tf[2][LEVEL];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 u[2], t[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int it = 2 * p + h;
          e[it] = y[it] - e[it];
          u[h] = e[it] * four(rec.beta + 16 * it + 4 * q4);
          t[h] = u[h] * four(rec.rk_to_end + 16 * it + 4 * q4);
        }
        if constexpr (!TOTALS) {
          bf16x8 uf[OUT];
          split8<OUT>(u[0], u[1], uf);
          store_frag<OUT>(Us, w * 2 + p, l, uf);
        }
        split8<LEVEL>(t[0], t[1], tf[p]);
      }
      const float times = rec.times, plus = rec.plus;
      lds_barrier();   // U and P are there, of the chunk K is needed yet
      if (!TOTALS && errors != nullptr) {
        float* to = errors + (size_t(unit) * chunks + c) * CHUNK * DV;
        const int ld = in_this_step(DV);
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + (16 * it + v) * ld)[at_token] = e[it][v];
      }
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) S[t][v] = __builtin_fmaf(S[t][v], plus, S[t][v] * times);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        constexpr int AT_ONCE = 2 * KS < 4 ? 2 * KS : 4;
#pragma unroll
        for (int t0 = 0; t0 < 2 * KS; t0 += AT_ONCE) {
          bf16x8 kf[AT_ONCE][IN];
#pragma unroll
          for (int t = 0; t < AT_ONCE; ++t)
            KTile::spread_col_frag(Ks, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of((t0 + t) / 2, (t0 + t) % 2, 0, 0), r, kf[t]);
          mm_each<LEVEL>(kf, tf[p], S + t0);
        }
      }
      lds_barrier();   // K and the updates are read
    }
    float* to = state_out != nullptr && ends_here ? state_out + size_t(unit) * DK * DV : nullptr;
    if (TOTALS) to = unit_columns ? transitions + (size_t(unit) * G.n + g) * DK * DK : starts + (size_t(unit) * G.n + g + 1) * DK * DV;
    if (to != nullptr && col0 + 16 * w < width) {
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * width)[at_key] = S[t][v];
    }
    return;
  }

  if (role == 1) {
    // ---- the chunks' rows
    constexpr int W_PIECES = (W_FRAGS * LEVEL * 64 + NT - 1) / NT, REC_PIECES = (RECORD_PIECES + NT - 1) / NT;
    const T* Qu = Q + size_t(unit) * N * DK;
    const T* Ku = K + size_t(unit) * N * DK;
    const T* Vu = V + size_t(unit) * N * DV + col0;
    RowTile<T, DK, 16, NT> kt, qt;
    RowTile<T, VC, 16, NT> vt;
    u32x4 rec_next[REC_PIECES], w_next[W_PIECES];
    const auto fetch = [&](int c) {
      const int row0 = c * CHUNK;
      const size_t at = size_t(unit) * chunks + c;
#pragma unroll
      for (int i = 0; i < REC_PIECES; ++i)
        if (i * NT + tid < RECORD_PIECES) rec_next[i] = reinterpret_cast<const u32x4*>(records + at)[i * NT + tid];
      if constexpr (!TOTALS) qt.fetch(Qu + size_t(row0) * DK, there - row0);
      if (Cfg::V_IN_LDS && !unit_columns) vt.fetch(Vu + size_t(row0) * DV, there - row0, DV);
#pragma unroll
      for (int i = 0; i < W_PIECES; ++i)
        if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64)
          w_next[i] = reinterpret_cast<const u32x4*>(w_rows + at * W_ELEMS)[i * NT + tid];
      kt.fetch(Ku + size_t(row0) * DK, there - row0);
    };
    const auto commit = [&]() {   // all but K
      if constexpr (!TOTALS) {
        qt.commit(Qs);
        qt.store_factors(rq, inv_eps);
      }
      if (Cfg::V_IN_LDS && !unit_columns) vt.commit(Vs);
#pragma unroll
      for (int i = 0; i < REC_PIECES; ++i)
        if (i * NT + tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[i * NT + tid] = rec_next[i];
#pragma unroll
      for (int i = 0; i < W_PIECES; ++i)
        if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64) reinterpret_cast<u32x4*>(Ws)[i * NT + tid] = w_next[i];
    };
    if (first < steps) {
      fetch(first);
      commit();
    }
    for (int c = first; c < steps; ++c) {
      kt.commit(Ks);
      lds_barrier();   // the chunk is there
      if (c + 1 < steps) fetch(c + 1);
      lds_barrier();   // of the chunk K is needed yet
      if (c + 1 < steps) commit();
      lds_barrier();   // K is read
    }
    return;
  }

  // ---- the results
  if constexpr (TOTALS) return;
  T* Ou = O + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  for (int c = first; c < steps; ++c) {
    const int row0 = c * CHUNK;
    lds_barrier();   // the chunk is there
    // P, a tile of rows to a wave (two where there are two waves), keys down: an operand as it stands.  (The tiles above the
    // diagonal, too: the workgroup waits for the wave that has none.)
#pragma unroll
    for (int turn = 0; turn < 4 / NW; ++turn) {
      const int it = turn == 0 ? w : 3 - w, own = 16 * it + r;
      f32x4 t[4];
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) t[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 qf[IN], kf[4][IN];
        KTile::row_frag(Qs, own, 32 * ks + 8 * q4, qf);
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) KTile::row_frag(Ks, 16 * jt + r, 32 * ks + 8 * q4, kf[jt]);
        mm_each<OUT>(kf, qf, t);
      }
      const float rq_own = rq[own], in_tile = rec.in_tile[own];
      f32x4 diagonal;
      {
        const double g_own = rec.decay[own];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int j = 16 * it + 4 * q4 + v;
          diagonal[v] = j <= own ? rec.rk[j] * decay_between(g_own, rec.decay[j]) : 0.f;
        }
      }
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) {
        const f32x4 below = four(rec.rk_to_tile + 16 * jt + 4 * q4) * (in_tile * rec.between[it][jt]);   // 0 from the diagonal on
        t[jt] *= rq_own;
#pragma unroll
        for (int v = 0; v < 4; ++v) t[jt][v] *= jt == it ? diagonal[v] : below[v];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (w_row_there(it, p)) {
          bf16x8 pf[OUT];
          split8<OUT>(t[2 * p], t[2 * p + 1], pf);
          store_frag<OUT>(Ps, w_row_frag(it, p), l, pf);
        }
    }
    f32x4 o[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 sf[OUT], qf[4][IN];
      load_frag(Ss, w * KS + ks, l, sf);
#pragma unroll
      for (int t = 0; t < 4; ++t) KTile::row_frag(Qs, 16 * t + r, 32 * ks + 8 * q4, qf[t]);
      mm_each<OUT>(sf, qf, o);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] *= rq[16 * t + r] * rec.since[16 * t + r];
    lds_barrier();   // U and P are there, of the chunk K is needed yet
    {
      bf16x8 uf[2][OUT], pf[4][OUT], pl[2][OUT];
      load_frag(Us, w * 2, l, uf[0]);
#pragma unroll
      for (int it = 0; it < 4; ++it) load_frag(Ps, w_row_frag(it, 0), l, pf[it]);
      load_frag(Us, w * 2 + 1, l, uf[1]);
#pragma unroll
      for (int it = 0; it < 2; ++it) load_frag(Ps, w_row_frag(2 + it, 1), l, pl[it]);
      mm_each<OUT>(uf[0], pf, o);
      mm_each<OUT>(uf[1], pl, o + 2);
    }
    if (O != nullptr) {
#pragma unroll
      for (int it = 0; it < 4; ++it)
        if (row0 + 16 * it + r < there)
          *reinterpret_cast<vec4*>(Ou + (size_t(row0) + 16 * it) * DV + unsigned(r * DV + 16 * w + 4 * q4)) =
              vec4{T(scale * o[it][0]), T(scale * o[it][1]), T(scale * o[it][2]), T(scale * o[it][3])};
    }
    lds_barrier();   // the updates and P are read
  }
  // rows that do not exist
  if (O == nullptr) return;
  const int lo = max(there, first * CHUNK), hi = min(N, (first + seg) * CHUNK);
  for (long i = tid; i < long(hi - lo) * (VC / 4); i += NT)
    *reinterpret_cast<vec4*>(Ou + size_t(lo + i / (VC / 4)) * DV + i % (VC / 4) * 4) = vec4{T(0.f), T(0.f), T(0.f), T(0.f)};
}

// The same by waves that do all of it, for rows of 128 in fp32, whose three parts leave the LDS no room for what one half of the
// waves hands the other, nor for rows of V.  (Two waves, dv = 32, take 512 registers and spill 33 of a lane.)
template <typename T, int DK, int NW>
struct DeltaWideFwdCfg {
  static_assert(sizeof(T) == 4 && DK == 128 && (NW == 2 || NW == 4), "the rows that the other scan has no room for");
  static constexpr int LEVEL = 3, IN = Rows<T>::PARTS, OUT = RESULT_LEVEL<T>, VC = 16 * NW;
  using KTile = PartTile<CHUNK, DK, IN>;
  static constexpr int W_SIZE = W_FRAGS * LEVEL * 512, P_SIZE = W_FRAGS * OUT * 512;
};

template <typename T, int DK, int NW>
__global__ __launch_bounds__(64 * NW, 1) void delta_wide_fwd_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* state_in, T* __restrict__ O, float* state_out,
    const ChunkRecord* __restrict__ records, const uint16_t* __restrict__ w_rows, float* __restrict__ errors,
    float* __restrict__ states, const float* __restrict__ starts, Divisor H, Divisor G, Divisor parts, int seg, int N, int units,
    int DV, float inv_eps) {
  using Cfg = DeltaWideFwdCfg<T, DK, NW>;
  using KTile = typename Cfg::KTile;
  constexpr int LEVEL = Cfg::LEVEL, IN = Cfg::IN, OUT = Cfg::OUT, KS = DK / 32, NT = 64 * NW, VC = Cfg::VC;
  constexpr int W_PIECES = (W_FRAGS * LEVEL * 64 + NT - 1) / NT, REC_PIECES = (RECORD_PIECES + NT - 1) / NT;
  typedef __attribute__((ext_vector_type(4))) T vec4;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[Cfg::W_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[Cfg::P_SIZE];
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK];
  fetch_argument_now(Q, K, V, s, lengths, state_in, O, state_out, records, w_rows, errors, states, starts, H, G, parts, seg, N, units, DV,
                     inv_eps);
  int unit, part, g = 0;
  if (G.n == 1) {
    unit_and_segment(blockIdx.x, units, parts, unit, part);
  } else {   // (blockIdx.y: the part)
    unit_and_segment(blockIdx.x, units, G, unit, g);
    part = blockIdx.y;
  }
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int there = valid_rows(lengths, unit, H, N), chunks = delta_chunks(N), all = delta_chunks(there), first = g * seg, steps = min(all, first + seg), col0 = part * VC;
  const bool ends_here = steps == all && (first < all || g == 0);   // the state after the last row
  const bool put_by = g == 0 && G.n > 1 && !ends_here && state_in != nullptr && state_in == state_out;
  const float* from = g == 0 && !put_by ? (state_in != nullptr ? state_in + size_t(unit) * DK * DV : nullptr) : starts + (size_t(unit) * G.n + g) * DK * DV;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* Vu = V + size_t(unit) * N * DV + col0;
  T* Ou = O + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  // this lane's value column in the first key row, and in the first token row, that it holds
  const unsigned at_key = unsigned(8 * q4 * DV + col0 + 16 * w + r), at_token = unsigned(4 * q4 * DV + col0 + 16 * w + r);

  f32x4 S[2 * KS];
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      S[t][v] = from != nullptr && (g == 0 || first < all) ? (from + key_of(t / 2, t % 2, 0, v) * DV)[at_key] : 0.f;

  RowTile<T, DK, 16, NT> kt, qt;
  f32x4 vraw[4];
  u32x4 rec_next[REC_PIECES], w_next[W_PIECES];
  const auto fetch = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku + size_t(row0) * DK, there - row0);
    qt.fetch(Qu + size_t(row0) * DK, there - row0);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int row = 16 * t + 4 * q4 + v;
        vraw[t][v] = 0.f;
        if (row0 + row < there) vraw[t][v] = (Vu + (size_t(row0) + 16 * t + v) * DV)[unsigned(4 * q4 * DV + 16 * w + r)];
      }
    const size_t at = size_t(unit) * chunks + c;
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) rec_next[i] = reinterpret_cast<const u32x4*>(records + at)[i * NT + tid];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64)
        w_next[i] = reinterpret_cast<const u32x4*>(w_rows + at * W_ELEMS)[i * NT + tid];
  };
  if (steps > first) fetch(first);
  for (int c = first; c < steps; ++c) {
    const int row0 = c * CHUNK;
    kt.commit(Ks);
    qt.commit(Qs);
    qt.store_factors(rq, inv_eps);
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[i * NT + tid] = rec_next[i];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64) reinterpret_cast<u32x4*>(Ws)[i * NT + tid] = w_next[i];
    f32x4 y[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = vraw[t];
    __syncthreads();
    if (c + 1 < steps) fetch(c + 1);
    if (states != nullptr) {
      float* to = states + (size_t(unit) * chunks + c) * DK * DV;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = S[t][v];
    }

    // what the state before the chunk gives: Kh H, and Qh H
    f32x4 kh[4], o[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) kh[t] = o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 sf[LEVEL], kf[4][IN], qf[4][IN];
      split8<LEVEL>(S[2 * ks], S[2 * ks + 1], sf);
#pragma unroll
      for (int t = 0; t < 4; ++t) KTile::row_frag(Ks, 16 * t + r, 32 * ks + 8 * q4, kf[t]);
#pragma unroll
      for (int t = 0; t < 4; ++t) KTile::row_frag(Qs, 16 * t + r, 32 * ks + 8 * q4, qf[t]);
#pragma unroll
      for (int t = 0; t < 4; ++t) kh[t] = mm<LEVEL>(kf[t], sf, kh[t]);
#pragma unroll
      for (int t = 0; t < 4; ++t) o[t] = mm<OUT>(sf, qf[t], o[t]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 yf[2][LEVEL];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const f32x4 since = *reinterpret_cast<const f32x4*>(rec.rk_since + 16 * t + 4 * q4);
#pragma unroll
      for (int v = 0; v < 4; ++v) y[t][v] = __builtin_fmaf(-since[v], kh[t][v], y[t][v]);
    }
    split8<LEVEL>(y[0], y[1], yf[0]);
    split8<LEVEL>(y[2], y[3], yf[1]);

    __builtin_amdgcn_sched_barrier(0);
    // P, a tile of rows to a wave (two where there are two waves), keys down: an operand as it stands
#pragma unroll
    for (int turn = 0; turn < 4 / NW; ++turn) {
      const int it = turn == 0 ? w : 3 - w, own = 16 * it + r;
      const float rq_own = rq[own];
      bf16x8 qf[KS][IN];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) KTile::row_frag(Qs, own, 32 * ks + 8 * q4, qf[ks]);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (!w_row_there(it, p)) break;
        f32x4 half[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int jt = 2 * p + h;
          if (jt > it) break;
          f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            bf16x8 kf[IN];
            KTile::row_frag(Ks, 16 * jt + r, 32 * ks + 8 * q4, kf);
            t = mm<OUT>(kf, qf[ks], t);
          }
          if (jt < it) {
            half[h] = t * *reinterpret_cast<const f32x4*>(rec.rk_to_tile + 16 * jt + 4 * q4) *
                      (rq_own * rec.in_tile[own] * rec.between[it][jt]);
          } else {
            const double g_own = rec.decay[own];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int j = 16 * jt + 4 * q4 + v;
              half[h][v] = j <= own ? t[v] * rec.rk[j] * (rq_own * decay_between(g_own, rec.decay[j])) : 0.f;
            }
          }
        }
        bf16x8 pf[OUT];
        split8<OUT>(half[0], half[1], pf);
#pragma unroll
        for (int i = 0; i < OUT; ++i)
          reinterpret_cast<u32x4*>(Ps)[(w_row_frag(it, p) * OUT + i) * 64 + l] = __builtin_bit_cast(u32x4, pf[i]);
      }
    }

    __builtin_amdgcn_sched_barrier(0);
    // the errors and the updates
    bf16x8 uf[2][OUT], tf[2][LEVEL];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x4 e[2], u[2], t[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int it = 2 * p + h;
        e[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k <= p; ++k) {
          bf16x8 wf[LEVEL];
#pragma unroll
          for (int i = 0; i < LEVEL; ++i)
            wf[i] = __builtin_bit_cast(bf16x8, reinterpret_cast<const u32x4*>(Ws)[(w_row_frag(it, k) * LEVEL + i) * 64 + l]);
          e[h] = mm<LEVEL>(wf, yf[k], e[h]);
        }
        e[h] = y[it] - e[h];
        u[h] = e[h] * *reinterpret_cast<const f32x4*>(rec.beta + 16 * it + 4 * q4);
        t[h] = u[h] * *reinterpret_cast<const f32x4*>(rec.rk_to_end + 16 * it + 4 * q4);
        if (errors != nullptr) {
          float* to = errors + (size_t(unit) * chunks + c) * CHUNK * DV;
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + (16 * it + v) * DV)[at_token] = e[h][v];
        }
      }
      split8<OUT>(u[0], u[1], uf[p]);
      split8<LEVEL>(t[0], t[1], tf[p]);
    }

    __builtin_amdgcn_sched_barrier(0);
    // the state behind the chunk
    const float times = rec.times, plus = rec.plus;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) {
#pragma unroll
      for (int v = 0; v < 4; ++v) S[t][v] = __builtin_fmaf(S[t][v], plus, S[t][v] * times);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x8 kf[IN];
        KTile::spread_col_frag(Ks, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, kf);
        S[t] = mm<LEVEL>(kf, tf[p], S[t]);
      }
    }
    __syncthreads();   // P is there

    // the rows' results
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      o[it] *= rq[16 * it + r] * rec.since[16 * it + r];
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (w_row_there(it, p)) {
          bf16x8 pf[OUT];
#pragma unroll
          for (int i = 0; i < OUT; ++i)
            pf[i] = __builtin_bit_cast(bf16x8, reinterpret_cast<const u32x4*>(Ps)[(w_row_frag(it, p) * OUT + i) * 64 + l]);
          o[it] = mm<OUT>(uf[p], pf, o[it]);
        }
      if (O != nullptr && row0 + 16 * it + r < there)
        *reinterpret_cast<vec4*>(Ou + (size_t(row0) + 16 * it) * DV + unsigned(r * DV + 16 * w + 4 * q4)) =
            vec4{T(scale * o[it][0]), T(scale * o[it][1]), T(scale * o[it][2]), T(scale * o[it][3])};
    }
    __syncthreads();   // everything of the chunk is read
  }
  if (state_out != nullptr && ends_here) {
    float* to = state_out + size_t(unit) * DK * DV;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = S[t][v];
  }
  // rows that do not exist
  if (O == nullptr) return;
  const int lo = max(there, first * CHUNK), hi = min(N, (first + seg) * CHUNK);
  for (long i = tid; i < long(hi - lo) * (VC / 4); i += NT)
    *reinterpret_cast<vec4*>(Ou + size_t(lo + i / (VC / 4)) * DV + i % (VC / 4) * 4) = vec4{T(0.f), T(0.f), T(0.f), T(0.f)};
}

template <typename T, int DK, int NW>
hipError_t run_scan(const DeltaArgs& a) {
  const int units = a.B * a.H, parts = a.dv / (16 * NW);
  const ChunkRecord* records = static_cast<const ChunkRecord*>(a.records);
  const auto grid = [&](int n_parts) { return a.G == 1 ? dim3(unsigned(units * n_parts)) : dim3(unsigned(units * a.G), unsigned(n_parts)); };
  const auto run = [&](auto kernel, int n_parts, int threads) {
    return launch_kernel("delta_fwd_scan", kernel, grid(n_parts), dim3(threads), 0, a.stream, static_cast<const T*>(a.Q),
                         static_cast<const T*>(a.K), static_cast<const T*>(a.V), a.s, a.seq_len, a.state_in, static_cast<T*>(a.O), a.state,
                         records, a.w_rows, a.errors, a.states, a.starts, a.transitions, Divisor(a.H), Divisor(a.G), Divisor(n_parts),
                         a.seg, a.N, units, a.dv, largest_factor(a.eps));
  };
  if (a.G > 1) {
    // M is for delta_carry, which runs where there are more than two segments.  (With two a call that a backward follows forms it as
    // well, and with more the last segment does: nothing reads those.)
    const int with_M = a.G > 2 || a.errors != nullptr ? (DK + 16 * NW - 1) / (16 * NW) : 0;
    hipError_t err = run(delta_fwd_scan<T, DK, NW, true>, parts + with_M, 128 * NW);
    if (err == hipSuccess && a.G > 2) err = launch_delta_carry(a, false);
    if (err != hipSuccess) return err;
  }
  if constexpr (DeltaFwdCfg<T, DK, NW>::FITS) {
    return run(delta_fwd_scan<T, DK, NW, false>, parts, 192 * NW);
  } else {
    return launch_kernel("delta_fwd_scan", delta_wide_fwd_scan<T, DK, NW>, grid(parts), dim3(64 * NW), 0, a.stream,
                         static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.V), a.s, a.seq_len,
                         a.state_in, static_cast<T*>(a.O), a.state, records, a.w_rows, a.errors, a.states, a.starts, Divisor(a.H),
                         Divisor(a.G), Divisor(parts), a.seg, a.N, units, a.dv, largest_factor(a.eps));
  }
}

template <typename T, int DK>
hipError_t run_shape(const DeltaArgs& a) {
  return a.dv == 32 ? run_scan<T, DK, 2>(a) : run_scan<T, DK, 4>(a);
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
