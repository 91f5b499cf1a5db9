// The gated delta rule, backward (formulas, precision: delta.h): a scan from the last chunk to the first that leaves Z and the
// gradient D with respect to the state behind every chunk; then, of all chunks at once, the gradients; then the sums for ds.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

// ---------------------------------------------------------------------------------------
// As in the forward scan a wave has 16 value columns, whose D, F and X never leave its registers: F = P^T dO' + (G_n/G) Kh D, Z =
// F - W^T (b F), and D in front of the chunk, one after the other.  What does not depend on D, P^T dO' and R = (G Qh)^T dO', is
// formed beside that, a chunk ahead, by as many waves more; and again as many fetch the rows.  8 x 12 heads of 1024 rows at 64 x 64
// take 55 us, formed for the same chunk and by the waves that fetch 66.  What bounds it is, as there, the chain: steps of 7500
// cycles in which vector instructions issue in 49 % of them, matrix instructions in 27.  (Twelve waves have 168 registers each; one to
// three of a lane are spilled.)
template <typename T, int DK, int NW>
struct DeltaAheadCfg {
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3, VC = 16 * NW, KS = DK / 32;
  using KTile = PartTile<CHUNK, DK, IN>;
  using GTile = PartTile<CHUNK, VC, IN>;      // rows of dO
  static constexpr int W_SIZE = W_FRAGS * LEVEL * 512;
  static constexpr int BYTES = 2 * (3 * KTile::SIZE + GTile::SIZE + 2 * W_SIZE) + 2 * int(sizeof(ChunkRecord)) + 4 * CHUNK +
                               NW * (4 + 2 * KS) * 1024;
  static constexpr bool FITS = BYTES <= 160 * 1024;
};

// Parts of s (G Qh)'s factors times rows of dO, slots of two accumulator tiles: the tokens 32 p + 4 q .., 32 p + 16 + 4 q ...
template <int LEVEL, int IN>
__device__ __forceinline__ void weighted_rows(const bf16x8 (&g)[IN], const float* rq, const float* since, float scale, int t0,
                                              bf16x8 (&out)[LEVEL]) {
  f32x4 lo, hi;
  join8<IN>(g, lo, hi);
  split8<LEVEL>(lo * (four(rq + t0) * (scale * four(since + t0))), hi * (four(rq + t0 + 16) * (scale * four(since + t0 + 16))), out);
}

// Segments as in the forward scan: TOTALS leaves what a segment makes of zeros (the last one: of dstate) in the place of the
// gradient with respect to the state in front of it.  Where dstate_in is to replace dstate, that walk puts dstate by.
template <typename T, int DK, int NW, bool TOTALS>
__global__ __launch_bounds__(192 * NW, NW <= 2 ? 1 : 3) void delta_ahead_rev_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ dO, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* dstate, float* dstate_in, const ChunkRecord* __restrict__ records,
    const uint16_t* __restrict__ w_cols, float* __restrict__ zs, float* __restrict__ dstates, float* ends, Divisor H,
    Divisor G, Divisor parts, int seg, int N, int units, int DV, float inv_eps) {
  using Cfg = DeltaAheadCfg<T, DK, NW>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, KS = Cfg::KS, NT = 64 * NW, VC = Cfg::VC;
  __shared__ __attribute__((aligned(16))) uint16_t K2[2][KTile::SIZE];   // of the chunks with even and with odd numbers
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Os[GTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[Cfg::W_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[Cfg::W_SIZE];
  __shared__ f32x4 Fs[NW * 4 * 64];         // P^T dO', tiles in accumulator order
  __shared__ f32x4 Rs[NW * 2 * KS * 64];    // R
  __shared__ ChunkRecord recs[2];
  __shared__ __attribute__((aligned(16))) float rq[CHUNK];
  fetch_argument_now(Q, K, dO, s, lengths, dstate, dstate_in, records, w_cols, zs, dstates, ends, H, G, parts, seg, N, units, DV,
                     inv_eps);
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
  const int col0 = part * VC;
  if ((first >= all && g > 0) || (TOTALS && g == 0)) return;
  const bool ends_here = steps == all;   // the last rows
  const bool put_by = ends_here && g > 0 && dstate != nullptr && dstate == dstate_in;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];

  // In step c the first waves take chunk c and the others form what they will need of chunk c - 1, from the one behind the last on.
  if (role == 0) {
    // ---- the gradients with respect to the states
    // this lane's value column in the first key row, and in the first token row, that it holds
    const unsigned at_key = unsigned(8 * q4 * DV + col0 + 16 * w + r), at_token = unsigned(4 * q4 * DV + col0 + 16 * w + r);
    const float* from = ends_here && (TOTALS || !put_by) ? (dstate != nullptr ? dstate + size_t(unit) * DK * DV : nullptr)
                        : TOTALS ? nullptr : ends + (size_t(unit) * G.n + g) * DK * DV;
    f32x4 D[2 * KS];
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        D[t][v] = from != nullptr ? (from + key_of(t / 2, t % 2, 0, v) * DV)[at_key] : 0.f;
    if (TOTALS && put_by) {
      float* to = ends + (size_t(unit) * G.n + g) * DK * DV;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
    }
    lds_barrier();
    lds_barrier();
    lds_barrier();
    for (int c = steps - 1; c >= first; --c) {
      const uint16_t* Ks = K2[c & 1];
      const ChunkRecord& rec = recs[c & 1];
      bf16x8 df[KS][LEVEL];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) split8<LEVEL>(D[2 * ks], D[2 * ks + 1], df[ks]);
      if constexpr (!TOTALS) {
        float* to = dstates + (size_t(unit) * chunks + c) * DK * DV;
        const int ld = in_this_step(DV);
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * ld)[at_key] = D[t][v];
      }
      lds_barrier();   // the chunk is there
      f32x4 f[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[4][IN];
#pragma unroll
        for (int t = 0; t < 4; ++t) KTile::row_frag(Ks, 16 * t + r, 32 * ks + 8 * q4, kf[t]);
        mm_each<LEVEL>(kf, df[ks], f);
      }
      f32x4 b[4], z[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f[t] = f[t] * four(rec.rk_to_end + 16 * t + 4 * q4) + Fs[(w * 4 + t) * 64 + l];
        b[t] = four(rec.beta + 16 * t + 4 * q4);
        z[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      bf16x8 ff[2][LEVEL], xf[2][LEVEL];
#pragma unroll
      for (int p = 0; p < 2; ++p) split8<LEVEL>(b[2 * p] * f[2 * p], b[2 * p + 1] * f[2 * p + 1], ff[p]);
      {
        bf16x8 wf[2][LEVEL], wl[4][LEVEL];
#pragma unroll
        for (int t = 0; t < 2; ++t) load_frag(Ws, w_col_frag(t, 0), l, wf[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) load_frag(Ws, w_col_frag(t, 1), l, wl[t]);
        mm_each<LEVEL>(wl, ff[1], z);
        mm_each<LEVEL>(wf, ff[0], z);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = 2 * p + h;
          z[t] = f[t] - z[t];
          x[h] = -(b[t] * z[t]) * four(rec.rk_since + 16 * t + 4 * q4);
        }
        split8<LEVEL>(x[0], x[1], xf[p]);
      }
      const float times = rec.times, plus = rec.plus;
      lds_barrier();   // of the chunk K is needed yet
      if constexpr (!TOTALS) {
        float* to = zs + (size_t(unit) * chunks + c) * CHUNK * DV;
        const int ld = in_this_step(DV);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + (16 * t + v) * ld)[at_token] = z[t][v];
      }
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) D[t][v] = __builtin_fmaf(D[t][v], plus, D[t][v] * times);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        constexpr int AT_ONCE = 2 * KS < 4 ? 2 * KS : 4;
#pragma unroll
        for (int t0 = 0; t0 < 2 * KS; t0 += AT_ONCE) {
          bf16x8 kf[AT_ONCE][IN];
#pragma unroll
          for (int t = 0; t < AT_ONCE; ++t)
            KTile::spread_col_frag(Ks, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of((t0 + t) / 2, (t0 + t) % 2, 0, 0), r, kf[t]);
          mm_each<LEVEL>(kf, xf[p], D + t0);
        }
      }
      lds_barrier();   // K is read, R is there
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t) D[t] += Rs[(w * 2 * KS + t) * 64 + l];
    }
    float* to = TOTALS ? ends + (size_t(unit) * G.n + g - 1) * DK * DV : dstate_in != nullptr && g == 0 ? dstate_in + size_t(unit) * DK * DV : nullptr;
    if (to != nullptr) {
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
    }
    return;
  }

  if (role == 1) {
    // ---- the chunks' rows
    constexpr int W_PIECES = (W_FRAGS * LEVEL * 64 + NT - 1) / NT, REC_PIECES = (RECORD_PIECES + NT - 1) / NT;
    const T* Qu = Q + size_t(unit) * N * DK;
    const T* Ku = K + size_t(unit) * N * DK;
    const T* dOu = dO + size_t(unit) * N * DV + col0;
    RowTile<T, DK, 16, NT> kt, qt;
    RowTile<T, VC, 16, NT> gt;
    u32x4 rec_next[REC_PIECES], w_next[W_PIECES];
    const auto fetch = [&](int c) {
      const int row0 = c * CHUNK;
#pragma unroll
      for (int i = 0; i < REC_PIECES; ++i)
        if (i * NT + tid < RECORD_PIECES) rec_next[i] = reinterpret_cast<const u32x4*>(records + size_t(unit) * chunks + c)[i * NT + tid];
      kt.fetch(Ku + size_t(row0) * DK, there - row0);
      qt.fetch(Qu + size_t(row0) * DK, there - row0);
      gt.fetch(dOu + size_t(row0) * DV, there - row0, DV);
    };
    const auto commit = [&](int c) {
      kt.commit(K2[c & 1]);
      qt.commit(Qs);
      qt.store_factors(rq, inv_eps);
      gt.commit(Os);
#pragma unroll
      for (int i = 0; i < REC_PIECES; ++i)
        if (i * NT + tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&recs[c & 1])[i * NT + tid] = rec_next[i];
    };
    const auto fetch_W = [&](int c) {
#pragma unroll
      for (int i = 0; i < W_PIECES; ++i)
        if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64)
          w_next[i] = reinterpret_cast<const u32x4*>(w_cols + (size_t(unit) * chunks + c) * W_ELEMS)[i * NT + tid];
    };
    if (steps > first) {
      fetch(steps - 1);
      fetch_W(steps - 1);
      commit(steps - 1);
    }
    for (int c = steps; c >= first; --c) {
      lds_barrier();   // the chunk in front is there
      if (c - 2 >= first) fetch(c - 2);
      lds_barrier();   // of the chunk K is needed yet
      if (c - 1 >= first) {
#pragma unroll
        for (int i = 0; i < W_PIECES; ++i)
          if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64) reinterpret_cast<u32x4*>(Ws)[i * NT + tid] = w_next[i];
      }
      if (c - 2 >= first) fetch_W(c - 2);
      lds_barrier();   // K is read, and the rows of the one in front
      if (c - 2 >= first) commit(c - 2);
    }
    return;
  }

  // ---- what a chunk comes to by itself
  f32x4 R[2 * KS];
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t) R[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int c = steps; c >= first; --c) {
    const uint16_t* Ks = K2[(c - 1) & 1];
    const ChunkRecord& rec = recs[(c - 1) & 1];
    lds_barrier();   // the chunk in front is there
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) Rs[(w * 2 * KS + t) * 64 + l] = R[t];
    if (c == first) {
      lds_barrier();
      lds_barrier();
      break;
    }
    // s P, a tile of columns to a wave (two where there are two waves), queries down: an operand as it stands.  (The tiles above
    // the diagonal, too: the workgroup waits for the wave that has none.)
#pragma unroll
    for (int turn = 0; turn < 4 / NW; ++turn) {
      const int jt = turn == 0 ? w : 3 - w, own = 16 * jt + r;
      f32x4 t[4];
#pragma unroll
      for (int it = 0; it < 4; ++it) t[it] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[IN], qf[4][IN];
        KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf);
#pragma unroll
        for (int it = 0; it < 4; ++it) KTile::row_frag(Qs, 16 * it + r, 32 * ks + 8 * q4, qf[it]);
        mm_each<LEVEL>(qf, kf, t);
      }
      f32x4 diagonal;
      {
        const double g_own = rec.decay[own];
        const float rk_own = scale * rec.rk[own];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int i = 16 * jt + 4 * q4 + v;
          diagonal[v] = i >= own ? rk_own * decay_between(rec.decay[i], g_own) : 0.f;
        }
      }
      const float to_tile = scale * rec.rk_to_tile[own];
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const f32x4 below = four(rec.in_tile + 16 * it + 4 * q4) * (to_tile * rec.between[it][jt]);   // 0 up to the diagonal
        t[it] *= four(rq + 16 * it + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) t[it][v] *= it == jt ? diagonal[v] : below[v];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (w_col_there(jt, p)) {
          bf16x8 pf[LEVEL];
          split8<LEVEL>(t[2 * p], t[2 * p + 1], pf);
          store_frag<LEVEL>(Ps, w_col_frag(jt, p), l, pf);
        }
    }
    bf16x8 gf[2][IN];
#pragma unroll
    for (int p = 0; p < 2; ++p) GTile::col_frag(Os, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * w, r, gf[p]);
    lds_barrier();   // P is there, and the sums of the chunk behind are taken
    {
      f32x4 f[4];
      bf16x8 pf[2][LEVEL], pl[4][LEVEL];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        load_frag(Ps, w_col_frag(t, 1), l, pl[t]);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) load_frag(Ps, w_col_frag(t, 0), l, pf[t]);
      mm_each<LEVEL>(pl, gf[1], f);
      mm_each<LEVEL>(pf, gf[0], f);
#pragma unroll
      for (int t = 0; t < 4; ++t) Fs[(w * 4 + t) * 64 + l] = f[t];
    }
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) R[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      bf16x8 wg[LEVEL];
      weighted_rows<LEVEL>(gf[p], rq, rec.since, scale, 32 * p + 4 * q4, wg);
      constexpr int AT_ONCE = 2 * KS < 4 ? 2 * KS : 4;
#pragma unroll
      for (int t0 = 0; t0 < 2 * KS; t0 += AT_ONCE) {
        bf16x8 qf[AT_ONCE][IN];
#pragma unroll
        for (int t = 0; t < AT_ONCE; ++t)
          KTile::spread_col_frag(Qs, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of((t0 + t) / 2, (t0 + t) % 2, 0, 0), r, qf[t]);
        mm_each<LEVEL>(qf, wg, R + t0);
      }
    }
    lds_barrier();   // the rows are read
  }
}

// Where the LDS has no room for a second chunk's K (fp16 at dk = 128, fp32 at 64): what does not depend on D formed for the same chunk, and by the waves that fetch
// the rows; R, where there is no room to hand it over, by the first waves.
template <typename T, int DK, int NW>
struct DeltaRevCfg {
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3, VC = 16 * NW, KS = DK / 32, PAD = sizeof(T) == 4 ? 8 : 16;
  using KTile = PartTile<CHUNK, DK, IN, PAD>;
  using GTile = PartTile<CHUNK, VC, IN, PAD>;      // rows of dO
  static constexpr int W_SIZE = W_FRAGS * LEVEL * 512;
  static constexpr int BYTES = 2 * (2 * KTile::SIZE + GTile::SIZE + 2 * W_SIZE) + int(sizeof(ChunkRecord)) + 4 * CHUNK + NW * 4 * 1024;
  static constexpr bool HANDS_R = BYTES + NW * 2 * KS * 1024 <= 160 * 1024;
  static constexpr bool FITS = BYTES <= 160 * 1024;
};

template <typename T, int DK, int NW, bool TOTALS>
__global__ __launch_bounds__(128 * NW, NW <= 2 ? 1 : 2) void delta_rev_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ dO, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* dstate, float* dstate_in, const ChunkRecord* __restrict__ records,
    const uint16_t* __restrict__ w_cols, float* __restrict__ zs, float* __restrict__ dstates, float* ends, Divisor H,
    Divisor G, Divisor parts, int seg, int N, int units, int DV, float inv_eps) {
  using Cfg = DeltaRevCfg<T, DK, NW>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, KS = Cfg::KS, NT = 64 * NW, VC = Cfg::VC;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Os[GTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[Cfg::W_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[Cfg::W_SIZE];
  __shared__ f32x4 Fs[NW * 4 * 64];                            // P^T dO', tiles in accumulator order
  __shared__ f32x4 Rs[Cfg::HANDS_R ? NW * 2 * KS * 64 : 1];    // (G Qh)^T dO'
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK];
  fetch_argument_now(Q, K, dO, s, lengths, dstate, dstate_in, records, w_cols, zs, dstates, ends, H, G, parts, seg, N, units, DV,
                     inv_eps);
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
  const int col0 = part * VC;
  if ((first >= all && g > 0) || (TOTALS && g == 0)) return;
  const bool ends_here = steps == all;   // the last rows
  const bool put_by = ends_here && g > 0 && dstate != nullptr && dstate == dstate_in;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];

  if (role == 0) {
    // ---- the gradients with respect to the states
    // this lane's value column in the first key row, and in the first token row, that it holds
    const unsigned at_key = unsigned(8 * q4 * DV + col0 + 16 * w + r), at_token = unsigned(4 * q4 * DV + col0 + 16 * w + r);
    const float* from = ends_here && (TOTALS || !put_by) ? (dstate != nullptr ? dstate + size_t(unit) * DK * DV : nullptr)
                        : TOTALS ? nullptr : ends + (size_t(unit) * G.n + g) * DK * DV;
    f32x4 D[2 * KS];
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        D[t][v] = from != nullptr ? (from + key_of(t / 2, t % 2, 0, v) * DV)[at_key] : 0.f;
    if (TOTALS && put_by) {
      float* to = ends + (size_t(unit) * G.n + g) * DK * DV;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
    }
    for (int c = steps - 1; c >= first; --c) {
      bf16x8 df[KS][LEVEL];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) split8<LEVEL>(D[2 * ks], D[2 * ks + 1], df[ks]);
      if constexpr (!TOTALS) {
        float* to = dstates + (size_t(unit) * chunks + c) * DK * DV;
        const int ld = in_this_step(DV);
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * ld)[at_key] = D[t][v];
      }
      lds_barrier();   // the chunk is there
      f32x4 f[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[4][IN];
#pragma unroll
        for (int t = 0; t < 4; ++t) KTile::row_frag(Ks, 16 * t + r, 32 * ks + 8 * q4, kf[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) f[t] = mm<LEVEL>(kf[t], df[ks], f[t]);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] *= four(rec.rk_to_end + 16 * t + 4 * q4);
      lds_barrier();   // P is there
      lds_barrier();   // P^T dO' is there
      bf16x8 ff[2][LEVEL], xf[2][LEVEL];
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] += Fs[(w * 4 + t) * 64 + l];
      f32x4 b[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) b[t] = four(rec.beta + 16 * t + 4 * q4);
#pragma unroll
      for (int p = 0; p < 2; ++p) split8<LEVEL>(b[2 * p] * f[2 * p], b[2 * p + 1] * f[2 * p + 1], ff[p]);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = 2 * p + h;
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (w_col_there(t, k)) {
              bf16x8 wf[LEVEL];
              load_frag(Ws, w_col_frag(t, k), l, wf);
              z = mm<LEVEL>(wf, ff[k], z);
            }
          z = f[t] - z;
          if constexpr (!TOTALS) {
            float* to = zs + (size_t(unit) * chunks + c) * CHUNK * DV;
            const int ld = in_this_step(DV);
#pragma unroll
            for (int v = 0; v < 4; ++v) (to + (16 * t + v) * ld)[at_token] = z[v];
          }
          x[h] = -(b[t] * z) * four(rec.rk_since + 16 * t + 4 * q4);
        }
        split8<LEVEL>(x[0], x[1], xf[p]);
      }
      const float times = rec.times, plus = rec.plus;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) D[t][v] = __builtin_fmaf(D[t][v], plus, D[t][v] * times);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x8 wg[LEVEL];
        if constexpr (!Cfg::HANDS_R) {
          bf16x8 gf[IN];
          GTile::col_frag(Os, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * w, r, gf);
          weighted_rows<LEVEL>(gf, rq, rec.since, scale, 32 * p + 4 * q4, wg);
        }
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) {
          bf16x8 kf[IN];
          KTile::spread_col_frag(Ks, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, kf);
          D[t] = mm<LEVEL>(kf, xf[p], D[t]);
          if constexpr (!Cfg::HANDS_R) {
            bf16x8 qf[IN];
            KTile::spread_col_frag(Qs, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, qf);
            D[t] = mm<LEVEL>(qf, wg, D[t]);
          }
        }
      }
      lds_barrier();   // everything of the chunk is read, and (G Qh)^T dO' is there
      if constexpr (Cfg::HANDS_R) {
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) D[t] += Rs[(w * 2 * KS + t) * 64 + l];
      }
    }
    float* to = TOTALS ? ends + (size_t(unit) * G.n + g - 1) * DK * DV : dstate_in != nullptr && g == 0 ? dstate_in + size_t(unit) * DK * DV : nullptr;
    if (to != nullptr) {
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
    }
    return;
  }

  // ---- the chunks' rows and what they come to by themselves
  constexpr int W_PIECES = (W_FRAGS * LEVEL * 64 + NT - 1) / NT, REC_PIECES = (RECORD_PIECES + NT - 1) / NT;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* dOu = dO + size_t(unit) * N * DV + col0;
  RowTile<T, DK, Cfg::PAD, NT> kt, qt;
  RowTile<T, VC, Cfg::PAD, NT> gt;
  u32x4 rec_next[REC_PIECES], w_next[W_PIECES];
  const auto fetch = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku + size_t(row0) * DK, there - row0);
    qt.fetch(Qu + size_t(row0) * DK, there - row0);
    gt.fetch(dOu + size_t(row0) * DV, there - row0, DV);
    const size_t at = size_t(unit) * chunks + c;
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) rec_next[i] = reinterpret_cast<const u32x4*>(records + at)[i * NT + tid];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64)
        w_next[i] = reinterpret_cast<const u32x4*>(w_cols + at * W_ELEMS)[i * NT + tid];
  };
  if (steps > first) fetch(steps - 1);
  for (int c = steps - 1; c >= first; --c) {
    kt.commit(Ks);
    qt.commit(Qs);
    qt.store_factors(rq, inv_eps);
    gt.commit(Os);
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[i * NT + tid] = rec_next[i];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64) reinterpret_cast<u32x4*>(Ws)[i * NT + tid] = w_next[i];
    lds_barrier();   // the chunk is there
    if (c > first) fetch(c - 1);

    // s P, a tile of columns to a wave (two where there are two waves), queries down: an operand as it stands
#pragma unroll
    for (int turn = 0; turn < 4 / NW; ++turn) {
      const int jt = turn == 0 ? w : 3 - w, own = 16 * jt + r;
      bf16x8 kf[KS][IN];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf[ks]);
      for (int p = 0; p < 2; ++p) {
        if (!w_col_there(jt, p)) continue;
        f32x4 half[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int it = 2 * p + h;
          if (it < jt) continue;
          f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            bf16x8 qf[IN];
            KTile::row_frag(Qs, 16 * it + r, 32 * ks + 8 * q4, qf);
            t = mm<LEVEL>(qf, kf[ks], t);
          }
          t *= four(rq + 16 * it + 4 * q4);
          if (it > jt) {
            half[h] = t * (four(rec.in_tile + 16 * it + 4 * q4) * (scale * rec.rk_to_tile[own] * rec.between[it][jt]));
          } else {
            const double g_own = rec.decay[own];
            const float rk_own = scale * rec.rk[own];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int i = 16 * it + 4 * q4 + v;
              half[h][v] = i >= own ? t[v] * (rk_own * decay_between(rec.decay[i], g_own)) : 0.f;
            }
          }
        }
        bf16x8 pf[LEVEL];
        split8<LEVEL>(half[0], half[1], pf);
        store_frag<LEVEL>(Ps, w_col_frag(jt, p), l, pf);
      }
    }
    bf16x8 gf[2][IN];
#pragma unroll
    for (int p = 0; p < 2; ++p) GTile::col_frag(Os, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * w, r, gf[p]);
    lds_barrier();   // P is there
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (w_col_there(t, p)) {
          bf16x8 pf[LEVEL];
          load_frag(Ps, w_col_frag(t, p), l, pf);
          f = mm<LEVEL>(pf, gf[p], f);
        }
      Fs[(w * 4 + t) * 64 + l] = f;
    }
    lds_barrier();   // P^T dO' is there
    if constexpr (Cfg::HANDS_R) {
      bf16x8 wg[2][LEVEL];
#pragma unroll
      for (int p = 0; p < 2; ++p) weighted_rows<LEVEL>(gf[p], rq, rec.since, scale, 32 * p + 4 * q4, wg[p]);
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          bf16x8 qf[IN];
          KTile::spread_col_frag(Qs, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, qf);
          x = mm<LEVEL>(qf, wg[p], x);
        }
        Rs[(w * 2 * KS + t) * 64 + l] = x;
      }
    }
    lds_barrier();   // everything of the chunk is read, and (G Qh)^T dO' is there
  }
}

// The same by waves that do all of it, where the LDS has no room for what one half of the waves hands the other: fp32 at dk = 128.
template <typename T, int DK, int NW>
struct DeltaWideRevCfg {
  static_assert(sizeof(T) == 4 && DK == 128 && NW == 2, "the rows that the other scans have no room for");
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3, VC = 16 * NW, PAD = 8;
  using KTile = PartTile<CHUNK, DK, IN, PAD>;
  using GTile = PartTile<CHUNK, VC, IN, PAD>;      // rows of dO
  static constexpr int W_SIZE = W_FRAGS * LEVEL * 512;
};

template <typename T, int DK, int NW, bool TOTALS>
__global__ __launch_bounds__(64 * NW, 1) void delta_wide_rev_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ dO, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* dstate, float* dstate_in, const ChunkRecord* __restrict__ records,
    const uint16_t* __restrict__ w_cols, float* __restrict__ zs, float* __restrict__ dstates, float* ends, Divisor H, Divisor G,
    Divisor parts, int seg, int N, int units, int DV, float inv_eps) {
  using Cfg = DeltaWideRevCfg<T, DK, NW>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, KS = DK / 32, NT = 64 * NW, VC = Cfg::VC;
  constexpr int W_PIECES = (W_FRAGS * LEVEL * 64 + NT - 1) / NT, REC_PIECES = (RECORD_PIECES + NT - 1) / NT;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Os[GTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[Cfg::W_SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[Cfg::W_SIZE];
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK];
  fetch_argument_now(Q, K, dO, s, lengths, dstate, dstate_in, records, w_cols, zs, dstates, ends, H, G, parts, seg, N, units, DV,
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
  if ((first >= all && g > 0) || (TOTALS && g == 0)) return;
  const bool ends_here = steps == all;   // the last rows
  const bool put_by = ends_here && g > 0 && dstate != nullptr && dstate == dstate_in;
  const float* from = ends_here && (TOTALS || !put_by) ? (dstate != nullptr ? dstate + size_t(unit) * DK * DV : nullptr)
                      : TOTALS ? nullptr : ends + (size_t(unit) * G.n + g) * DK * DV;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* dOu = dO + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  // this lane's value column in the first key row, and in the first token row, that it holds
  const unsigned at_key = unsigned(8 * q4 * DV + col0 + 16 * w + r), at_token = unsigned(4 * q4 * DV + col0 + 16 * w + r);

  f32x4 D[2 * KS];
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      D[t][v] = from != nullptr ? (from + key_of(t / 2, t % 2, 0, v) * DV)[at_key] : 0.f;
  if (TOTALS && put_by) {
    float* to = ends + (size_t(unit) * G.n + g) * DK * DV;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
  }

  RowTile<T, DK, Cfg::PAD, NT> kt, qt;
  RowTile<T, VC, Cfg::PAD, NT> gt;
  u32x4 rec_next[REC_PIECES], w_next[W_PIECES];
  const auto fetch = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku + size_t(row0) * DK, there - row0);
    qt.fetch(Qu + size_t(row0) * DK, there - row0);
    gt.fetch(dOu + size_t(row0) * DV, there - row0, DV);
    const size_t at = size_t(unit) * chunks + c;
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) rec_next[i] = reinterpret_cast<const u32x4*>(records + at)[i * NT + tid];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64)
        w_next[i] = reinterpret_cast<const u32x4*>(w_cols + at * W_ELEMS)[i * NT + tid];
  };
  if (steps > first) fetch(steps - 1);
  for (int c = steps - 1; c >= first; --c) {
    kt.commit(Ks);
    qt.commit(Qs);
    qt.store_factors(rq, inv_eps);
    gt.commit(Os);
#pragma unroll
    for (int i = 0; i < REC_PIECES; ++i)
      if (i * NT + tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[i * NT + tid] = rec_next[i];
#pragma unroll
    for (int i = 0; i < W_PIECES; ++i)
      if (W_FRAGS * LEVEL * 64 % NT == 0 || i * NT + tid < W_FRAGS * LEVEL * 64) reinterpret_cast<u32x4*>(Ws)[i * NT + tid] = w_next[i];
    __syncthreads();
    if (c > first) fetch(c - 1);
    if constexpr (!TOTALS) {
      float* to = dstates + (size_t(unit) * chunks + c) * DK * DV;
#pragma unroll
      for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
    }

    // s P, a tile of columns to a wave (two where there are two waves), queries down: an operand as it stands
#pragma unroll
    for (int turn = 0; turn < 4 / NW; ++turn) {
      const int jt = turn == 0 ? w : 3 - w, own = 16 * jt + r;
      bf16x8 kf[KS][IN];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf[ks]);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (!w_col_there(jt, p)) continue;
        f32x4 half[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int it = 2 * p + h;
          if (it < jt) continue;
          f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            bf16x8 qf[IN];
            KTile::row_frag(Qs, 16 * it + r, 32 * ks + 8 * q4, qf);
            t = mm<LEVEL>(qf, kf[ks], t);
          }
          t *= *reinterpret_cast<const f32x4*>(rq + 16 * it + 4 * q4);
          if (it > jt) {
            half[h] = t * (*reinterpret_cast<const f32x4*>(rec.in_tile + 16 * it + 4 * q4) *
                           (scale * rec.rk_to_tile[own] * rec.between[it][jt]));
          } else {
            const double g_own = rec.decay[own];
            const float rk_own = scale * rec.rk[own];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int i = 16 * it + 4 * q4 + v;
              half[h][v] = i >= own ? t[v] * (rk_own * decay_between(rec.decay[i], g_own)) : 0.f;
            }
          }
        }
        bf16x8 pf[LEVEL];
        split8<LEVEL>(half[0], half[1], pf);
#pragma unroll
        for (int i = 0; i < LEVEL; ++i)
          reinterpret_cast<u32x4*>(Ps)[(w_col_frag(jt, p) * LEVEL + i) * 64 + l] = __builtin_bit_cast(u32x4, pf[i]);
      }
    }

    // F: what D gives, and the chunk's own rows
    f32x4 f[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) f[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 df[LEVEL];
      split8<LEVEL>(D[2 * ks], D[2 * ks + 1], df);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        bf16x8 kf[IN];
        KTile::row_frag(Ks, 16 * t + r, 32 * ks + 8 * q4, kf);
        f[t] = mm<LEVEL>(kf, df, f[t]);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) f[t] *= *reinterpret_cast<const f32x4*>(rec.rk_to_end + 16 * t + 4 * q4);
    bf16x8 gf[2][IN];
#pragma unroll
    for (int p = 0; p < 2; ++p) GTile::col_frag(Os, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * w, r, gf[p]);
    __syncthreads();   // P is there
    const auto fragment = [&](const uint16_t* from, int tile, int p, bf16x8 (&x)[LEVEL]) {
#pragma unroll
      for (int i = 0; i < LEVEL; ++i)
        x[i] = __builtin_bit_cast(bf16x8, reinterpret_cast<const u32x4*>(from)[(w_col_frag(tile, p) * LEVEL + i) * 64 + l]);
    };
    bf16x8 ff[2][LEVEL], xf[2][LEVEL];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (w_col_there(t, p)) {
          bf16x8 pf[LEVEL];
          fragment(Ps, t, p, pf);
          f[t] = mm<LEVEL>(pf, gf[p], f[t]);
        }
    f32x4 b[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) b[t] = *reinterpret_cast<const f32x4*>(rec.beta + 16 * t + 4 * q4);
#pragma unroll
    for (int p = 0; p < 2; ++p) split8<LEVEL>(b[2 * p] * f[2 * p], b[2 * p + 1] * f[2 * p + 1], ff[p]);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x4 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = 2 * p + h;
        f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (w_col_there(t, k)) {
            bf16x8 wf[LEVEL];
            fragment(Ws, t, k, wf);
            z = mm<LEVEL>(wf, ff[k], z);
          }
        z = f[t] - z;
        if constexpr (!TOTALS) {
          float* to = zs + (size_t(unit) * chunks + c) * CHUNK * DV;
#pragma unroll
          for (int v = 0; v < 4; ++v) (to + (16 * t + v) * DV)[at_token] = z[v];
        }
        x[h] = -(b[t] * z) * *reinterpret_cast<const f32x4*>(rec.rk_since + 16 * t + 4 * q4);
      }
      split8<LEVEL>(x[0], x[1], xf[p]);
    }

    // D in front of the chunk
    bf16x8 wg[2][LEVEL];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x4 lo, hi;
      join8<IN>(gf[p], lo, hi);
      const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
      lo *= *reinterpret_cast<const f32x4*>(rq + t0) * (scale * *reinterpret_cast<const f32x4*>(rec.since + t0));
      hi *= *reinterpret_cast<const f32x4*>(rq + t1) * (scale * *reinterpret_cast<const f32x4*>(rec.since + t1));
      split8<LEVEL>(lo, hi, wg[p]);
    }
    const float times = rec.times, plus = rec.plus;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t) {
#pragma unroll
      for (int v = 0; v < 4; ++v) D[t][v] = __builtin_fmaf(D[t][v], plus, D[t][v] * times);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x8 kf[IN], qf[IN];
        KTile::spread_col_frag(Ks, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, kf);
        KTile::spread_col_frag(Qs, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, key_of(t / 2, t % 2, 0, 0), r, qf);
        D[t] = mm<LEVEL>(kf, xf[p], D[t]);
        D[t] = mm<LEVEL>(qf, wg[p], D[t]);
      }
    }
    __syncthreads();   // everything of the chunk is read
  }
  float* to = TOTALS ? ends + (size_t(unit) * G.n + g - 1) * DK * DV : dstate_in != nullptr && g == 0 ? dstate_in + size_t(unit) * DK * DV : nullptr;
  if (to != nullptr) {
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) (to + key_of(t / 2, t % 2, 0, v) * DV)[at_key] = D[t][v];
  }
}

// ---------------------------------------------------------------------------------------
// The gradients of a chunk, a workgroup each.  A wave owns key columns of dQ and dK, so that it meets, and takes apart, its rows
// of H and D once (twice where there are more waves than key tiles); accumulators hold them transposed, four consecutive columns of
// a token in a lane.  16 heads of 32768 rows at 64 x 64 take 306 us: HBM moves 621 MB (2.0 TB/s), the LDS 43 % of the time (39 % of
// that lanes that want the same bank), vector instructions issue in 39 %: phases with barriers between them, two workgroups to a
// compute unit.  Where the LDS holds but one, eight waves share it: 8 x 12 heads of 1024 rows at 128 x 128 177 -> 165 us, 32 heads
// in fp32 72 -> 64; two workgroups of eight waves have 128 registers, too few (64 x 64: 60 -> 68).  (bf16 at 128 x 64 spills eight
// of 256.)
template <typename T, int DK, int DV>
struct DeltaGradCfg {
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3, PAD = 8;
  using KTile = PartTile<CHUNK, DK, IN, PAD>;
  using GTile = PartTile<CHUNK, DV, IN, PAD>;
  using ETile = PartTile<CHUNK, DV, LEVEL, PAD>;
  using MTile = PartTile<CHUNK, CHUNK, LEVEL, PAD>;
  // first the rows of dO, E and Z, then two masked tiles and the rows of K and Q
  static constexpr int FIRST = GTile::SIZE + 2 * ETile::SIZE, SECOND = 2 * MTile::SIZE + 2 * KTile::SIZE;
  static constexpr int SIZE = FIRST > SECOND ? FIRST : SECOND;
  static constexpr int LDS_BYTES = 2 * SIZE + CHUNK * 8 + 32 + int(sizeof(ChunkRecord));
  static constexpr int GROUPS = (160 * 1024) / LDS_BYTES >= 2 ? 2 : 1;
  // key tiles, one to a wave, and token tiles that it forms of them
  static constexpr int WAVES = GROUPS == 2 ? 4 : 8, THREADS = 64 * WAVES, KT = DK / 16, NTOK = 4 * KT / WAVES;
  static_assert(WAVES % KT == 0, "a key tile to a wave");
};

template <typename T, int DK, int DV>
__global__ __launch_bounds__((DeltaGradCfg<T, DK, DV>::THREADS), (DeltaGradCfg<T, DK, DV>::WAVES / 4 * DeltaGradCfg<T, DK, DV>::GROUPS)) void delta_gradients(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const float* __restrict__ s, const float* __restrict__ log_decay, const float* __restrict__ beta,
    const int* __restrict__ lengths, const ChunkRecord* __restrict__ records, const float* __restrict__ errors,
    const float* __restrict__ states, const float* __restrict__ zs, const float* __restrict__ dstates, T* __restrict__ dQ,
    T* __restrict__ dK, T* __restrict__ dV, float* __restrict__ dlog_decay, float* __restrict__ dbeta,
    float* __restrict__ ds_parts, Divisor H, Divisor chunks, int N, float inv_eps, float below_eps, int from_state) {
  using Cfg = DeltaGradCfg<T, DK, DV>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  using ETile = typename Cfg::ETile;
  using MTile = typename Cfg::MTile;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, NTOK = Cfg::NTOK, VS = DV / 32, THREADS = Cfg::THREADS, KT = Cfg::KT;
  __shared__ __attribute__((aligned(16))) uint16_t room[Cfg::SIZE];
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK], xv[CHUNK];
  __shared__ float tail[Cfg::WAVES];
  typedef float Dots[KT][CHUNK];
  Dots& qdot = *reinterpret_cast<Dots*>(room);   // when nothing else is there any more
  Dots& kdot = *(&qdot + 1);
  uint16_t* const Os = room;
  uint16_t* const Es = Os + GTile::SIZE;
  uint16_t* const Zs = Es + ETile::SIZE;
  uint16_t* const Ms = room;                  // rows i, columns j, times the factor of row j
  uint16_t* const Mt = Ms + MTile::SIZE;      // the same times the factor of row i, read down its columns
  uint16_t* const Ks = Mt + MTile::SIZE;
  uint16_t* const Qs = Ks + KTile::SIZE;
  const int unit = quotient(blockIdx.x, chunks), c = blockIdx.x - unit * chunks.n, row0 = c * CHUNK;
  const int there = valid_rows(lengths, unit, H, N);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const size_t row_at = size_t(unit) * N;
  T* dQu = dQ + row_at * DK;
  T* dKu = dK + row_at * DK;
  T* dVu = dV + row_at * DV;
  {   // rows that do not exist
    typedef __attribute__((ext_vector_type(4))) T vec4;
    const vec4 none = {T(0.f), T(0.f), T(0.f), T(0.f)};
    const int lo = max(row0, there), hi = min(N, row0 + CHUNK);
    for (int i = tid; i < (hi - lo) * (DK / 4); i += THREADS) {
      *reinterpret_cast<vec4*>(dQu + size_t(lo) * DK + i * 4) = none;
      *reinterpret_cast<vec4*>(dKu + size_t(lo) * DK + i * 4) = none;
    }
    for (int i = tid; i < (hi - lo) * (DV / 4); i += THREADS) *reinterpret_cast<vec4*>(dVu + size_t(lo) * DV + i * 4) = none;
    if (tid < hi - lo) {
      dbeta[row_at + lo + tid] = 0.f;
      if (dlog_decay != nullptr) dlog_decay[row_at + lo + tid] = 0.f;
    }
  }
  if (row0 >= there) {
    if (tid == 0) ds_parts[blockIdx.x] = 0.f;
    return;
  }
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  // wave w: key tile kt0, token tiles tt0 .. tt0 + NTOK - 1
  const int kt0 = w % KT, tt0 = w / KT * NTOK;
  f32x4 hd[4];   // eight values of a key's row of H, and of D, 32 columns ahead
  const auto fetch_states = [&](int vs) {
    const size_t at = size_t(blockIdx.x) * DK * DV + size_t(16 * kt0 + r) * DV + 32 * vs + 8 * q4;
    hd[0] = reinterpret_cast<const f32x4*>(states + at)[0];
    hd[1] = reinterpret_cast<const f32x4*>(states + at)[1];
    hd[2] = reinterpret_cast<const f32x4*>(dstates + at)[0];
    hd[3] = reinterpret_cast<const f32x4*>(dstates + at)[1];
  };
  RowTile<T, DK, Cfg::PAD, THREADS> kt, qt;
  {
    using RT = RowTile<T, DV, Cfg::PAD, THREADS>;
    RT gt, vt;
    gt.fetch(dO + (row_at + row0) * DV, there - row0);
    vt.fetch(V + (row_at + row0) * DV, there - row0);
    kt.fetch(K + (row_at + row0) * DK, there - row0);
    qt.fetch(Q + (row_at + row0) * DK, there - row0);
    if (tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[tid] = reinterpret_cast<const u32x4*>(records + blockIdx.x)[tid];
    f32x4 ez[RT::PASSES][4];
    float b_row[RT::PASSES];
#pragma unroll
    for (int p = 0; p < RT::PASSES; ++p) {
      if (!RT::in(p)) continue;   // (whole waves)
      const size_t at = (size_t(blockIdx.x) * CHUNK + RT::row(p)) * DV + RT::col();
      ez[p][0] = reinterpret_cast<const f32x4*>(errors + at)[0];
      ez[p][1] = reinterpret_cast<const f32x4*>(errors + at)[1];
      ez[p][2] = reinterpret_cast<const f32x4*>(zs + at)[0];
      ez[p][3] = reinterpret_cast<const f32x4*>(zs + at)[1];
      b_row[p] = row0 + RT::row(p) < there ? beta[row_at + row0 + RT::row(p)] : 0.f;
    }
    fetch_states(0);
    gt.commit(Os);
#pragma unroll
    for (int p = 0; p < RT::PASSES; ++p) {
      if (!RT::in(p)) continue;
      const int row = RT::row(p), col = RT::col();
      const f32x4 e0 = ez[p][0], e1 = ez[p][1], z0 = ez[p][2], z1 = ez[p][3];
      const float b = b_row[p];
      bf16x8 parts[LEVEL];
      split8<LEVEL>(e0, e1, parts);
      ETile::store8(Es, row, col, parts);
      split8<LEVEL>(z0, z1, parts);
      ETile::store8(Zs, row, col, parts);
      f32x4 v0, v1;
      vt.raw[p].values(v0, v1);
      float ez = 0.f, zv = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ez = __builtin_fmaf(e0[i], z0[i], __builtin_fmaf(e1[i], z1[i], ez));
        zv = __builtin_fmaf(v0[i], z0[i], __builtin_fmaf(v1[i], z1[i], zv));
      }
      ez = group_sum<RT::LPR>(ez);
      zv = group_sum<RT::LPR>(zv);
      if (tid % RT::LPR == 0) xv[row] = b * zv;
      if (row0 + row < there) {
        if (tid % RT::LPR == 0) dbeta[row_at + row0 + row] = ez;
        typedef __attribute__((ext_vector_type(4))) T vec4;
        vec4* to = reinterpret_cast<vec4*>(dVu + size_t(row0 + row) * DV + col);
        to[0] = vec4{T(b * z0[0]), T(b * z0[1]), T(b * z0[2]), T(b * z0[3])};
        to[1] = vec4{T(b * z1[0]), T(b * z1[1]), T(b * z1[2]), T(b * z1[3])};
      }
    }
    qt.store_factors(rq, inv_eps);
  }
  __syncthreads();

  f32x4 aq[NTOK], ak[NTOK], az[NTOK];
  float through = 0.f;   // <D, H>, of the wave's rows
  {
#pragma unroll
    for (int t = 0; t < NTOK; ++t) aq[t] = ak[t] = az[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int vs = 0; vs < VS; ++vs) {
      const f32x4 h0 = hd[0], h1 = hd[1], d0 = hd[2], d1 = hd[3];
      if (vs + 1 < VS) fetch_states(vs + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) through = __builtin_fmaf(h0[i], d0[i], __builtin_fmaf(h1[i], d1[i], through));
      bf16x8 hf[LEVEL], df[LEVEL];
      split8<LEVEL>(h0, h1, hf);
      split8<LEVEL>(d0, d1, df);
#pragma unroll
      for (int t = 0; t < NTOK; ++t) {
        const int row = 16 * (tt0 + t) + r, col = 32 * vs + 8 * q4;
        bf16x8 gf[IN], ef[LEVEL], zf[LEVEL];
        GTile::row_frag(Os, row, col, gf);
        ETile::row_frag(Es, row, col, ef);
        ETile::row_frag(Zs, row, col, zf);
        aq[t] = mm<LEVEL>(hf, gf, aq[t]);
        ak[t] = mm<LEVEL>(df, ef, ak[t]);
        az[t] = mm<LEVEL>(hf, zf, az[t]);
      }
    }
    // each token's factors
#pragma unroll
    for (int t = 0; t < NTOK; ++t) {
      const int i = 16 * (tt0 + t) + r;
      const float since = rec.since[i], to_end = rec.beta[i] * decay_between(rec.decay[CHUNK - 1], rec.decay[i]);
      aq[t] *= since;
      ak[t] *= to_end;
      az[t] *= -rec.beta[i] * since;
    }
  }

  // the masked tiles: rows i of tile w % 4, columns j of all tiles or of every other one; lanes hold four columns of a row
  constexpr int APART = Cfg::WAVES / 4, TILES = 4 / APART;
  f32x4 pt[TILES], at[TILES];
  const int it = w % 4, jt0 = w / 4, own = 16 * it + r;
  const double g_own = rec.decay[own];
  const float b_own = rec.beta[own];
#pragma unroll
  for (int u = 0; u < TILES; ++u) pt[u] = at[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int vs = 0; vs < VS; ++vs) {
    bf16x8 gf[IN], zf[LEVEL];
    GTile::row_frag(Os, own, 32 * vs + 8 * q4, gf);
    ETile::row_frag(Zs, own, 32 * vs + 8 * q4, zf);
#pragma unroll
    for (int u = 0; u < TILES; ++u)
      if (jt0 + APART * u <= it) {
        bf16x8 ef[LEVEL];
        ETile::row_frag(Es, 16 * (jt0 + APART * u) + r, 32 * vs + 8 * q4, ef);
        pt[u] = mm<LEVEL>(ef, gf, pt[u]);
        at[u] = mm<LEVEL>(ef, zf, at[u]);
      }
  }
#pragma unroll
  for (int u = 0; u < TILES; ++u)
    if (jt0 + APART * u <= it) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int j = 16 * (jt0 + APART * u) + 4 * q4 + v;
        const float f = rec.beta[j] * decay_between(g_own, rec.decay[j]);
        pt[u][v] = j <= own ? pt[u][v] * f : 0.f;
        at[u][v] = j < own ? -b_own * at[u][v] * f : 0.f;
      }
    }
  const float rq_own = rq[own], rk_own = rec.rk[own];
  const auto store_masked = [&](const f32x4 (&m)[TILES], float by_row, bool zeros) {
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
      const int jt = jt0 + APART * u, j = 16 * jt + 4 * q4;
      if (jt <= it) {
        MTile::store4(Ms, own, j, m[u] * four(rec.rk + j));
        MTile::store4(Mt, own, j, m[u] * by_row);
      } else if (zeros && jt == (it | 1)) {   // (of the tiles above the diagonal the products read those beside it)
        MTile::store4(Ms, own, j, f32x4{0.f, 0.f, 0.f, 0.f});
        MTile::store4(Mt, own, j, f32x4{0.f, 0.f, 0.f, 0.f});
      }
    }
  };
  __syncthreads();   // the rows of dO, E and Z are read
  kt.commit(Ks);
  qt.commit(Qs);
  store_masked(pt, scale * rq_own, true);
  __syncthreads();
  // <D, H behind the chunk>: what goes through it, and what its updates give
  if (w >= KT) through = 0.f;   // (another wave has the same rows)
  through *= rec.since[CHUNK - 1];
#pragma unroll
  for (int t = 0; t < NTOK; ++t) {
    const int i = 16 * (tt0 + t) + r;
    float dot = 0.f;
    const f32x4 k = KTile::row4(Ks, i, 16 * kt0 + 4 * q4);
#pragma unroll
    for (int v = 0; v < 4; ++v) dot = __builtin_fmaf(k[v], ak[t][v], dot);
    ak[t] += az[t];
    through = __builtin_fmaf(rec.rk[i], dot, through);
  }
  through = group_sum<64>(through);
  if (l == 0) tail[w] = through;
#pragma unroll
  for (int round = 0; round < 2; ++round) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int t0 = 32 * ks + 8 * q4;
      bf16x8 kf[IN], qf[IN];
      KTile::col_frag(Ks, t0, t0 + 4, 16 * kt0, r, kf);
      if (round == 0) KTile::col_frag(Qs, t0, t0 + 4, 16 * kt0, r, qf);
#pragma unroll
      for (int t = 0; t < NTOK; ++t) {
        const int tt = tt0 + t;
        const bool before = 2 * ks <= tt, after = 2 * ks + 1 >= tt;   // columns up to row tt's tile; rows from column tt's tile on
        bf16x8 m[LEVEL];
        if (before) {
          MTile::row_frag(Ms, 16 * tt + r, t0, m);
          if (round == 0) aq[t] = mm<LEVEL>(kf, m, aq[t]);
          else ak[t] = mm<LEVEL>(kf, m, ak[t]);
        }
        if (after) {
          MTile::col_frag(Mt, t0, t0 + 4, 16 * tt, r, m);
          if (round == 0) ak[t] = mm<LEVEL>(qf, m, ak[t]);
          else ak[t] = mm<LEVEL>(kf, m, ak[t]);
        }
      }
    }
    if (round == 0) {
      __syncthreads();
      store_masked(at, rk_own, false);
      __syncthreads();
    }
  }

  __syncthreads();
  // through the normalisation: dq = (dqh - qh (qh . dqh)) / |q|; a row below eps was divided by eps alone
#pragma unroll
  for (int t = 0; t < NTOK; ++t) {
    const int i = 16 * (tt0 + t) + r;
    float dq = 0.f, dk = 0.f;
    const f32x4 q = KTile::row4(Qs, i, 16 * kt0 + 4 * q4), k = KTile::row4(Ks, i, 16 * kt0 + 4 * q4);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      dq = __builtin_fmaf(q[v], aq[t][v], dq);
      dk = __builtin_fmaf(k[v], ak[t][v], dk);
    }
    dq += __shfl_xor(dq, 16, 64);
    dk += __shfl_xor(dk, 16, 64);
    dq += __shfl_xor(dq, 32, 64);
    dk += __shfl_xor(dk, 32, 64);
    if (q4 == 0) {
      qdot[kt0][i] = dq;
      kdot[kt0][i] = dk;
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < NTOK; ++t) {
    const int i = 16 * (tt0 + t) + r;
    float dq = 0.f, dk = 0.f;
#pragma unroll
    for (int n = 0; n < KT; ++n) {
      dq += qdot[n][i];
      dk += kdot[n][i];
    }
    float fq = rq[i], fk = rec.rk[i];
    const float cq = fq == inv_eps ? 0.f : fq * (fq * dq), ck = fk == inv_eps ? 0.f : fk * (fk * dk);
    fq = fq == inv_eps ? below_eps : fq;
    fk = fk == inv_eps ? below_eps : fk;
    if (row0 + i < there) {
      const size_t at_ = size_t(row0 + i) * DK + 16 * kt0 + 4 * q4;
      const f32x4 q = KTile::row4(Qs, i, 16 * kt0 + 4 * q4), k = KTile::row4(Ks, i, 16 * kt0 + 4 * q4);
      typedef __attribute__((ext_vector_type(4))) T vec4;
      vec4 gq, gk;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        gq[v] = T(scale * (fq * __builtin_fmaf(-cq, q[v], aq[t][v])));
        gk[v] = T(fk * __builtin_fmaf(-ck, k[v], ak[t][v]));
      }
      *reinterpret_cast<vec4*>(dQu + at_) = gq;
      *reinterpret_cast<vec4*>(dKu + at_) = gk;
    }
  }
  if (w == 0) {   // lane l: token l
    float dot = 0.f;
#pragma unroll
    for (int n = 0; n < KT; ++n) dot += qdot[n][l];
    dot *= rq[l];   // qh . dqh / s
    const float sum = group_sum<64>(dot);
    if (l == 0) ds_parts[blockIdx.x] = sum;
    if (dlog_decay != nullptr) {
      double flow = double(scale * dot) - double(xv[l]);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double behind = __shfl_down(flow, d, 64);
        if (l + d < 64) flow += behind;
      }
#pragma unroll
      for (int n = 0; n < Cfg::WAVES; ++n) flow += double(tail[n]);
      if (row0 + l < there) {
        const float ld = log_decay[row_at + row0 + l];
        // 0 where the decay does not depend on it, or there is nothing yet to decay
        const bool none = ld > 0.f || ld < -128.f || (row0 + l == 0 && !from_state);
        dlog_decay[row_at + row0 + l] = none ? 0.f : float(flow);
      }
    }
  }
}

// ds[out] = the sum of its units' parts, in 64 bits, always in the same order: a wave each.  Without lengths the units are those
// of a head, `heads` apart.
__global__ __launch_bounds__(256) void delta_sum_ds(const float* __restrict__ parts, float* __restrict__ ds, int outs, int heads,
                                                    int units, int chunks) {
  const int out = blockIdx.x * 4 + int(threadIdx.x) / 64, l = threadIdx.x % 64;
  if (out >= outs) return;
  double sum = 0.0;
  for (long unit = out; unit < units; unit += heads)
    for (int c = l; c < chunks; c += 64) sum += double(parts[unit * chunks + c]);
#pragma unroll
  for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d, 64);
  if (l == 0) ds[out] = float(sum);
}

template <typename T, int DK, int NW>
hipError_t run_rev(const DeltaArgs& a) {
  const int units = a.B * a.H, parts = a.dv / (16 * NW);
  const ChunkRecord* records = static_cast<const ChunkRecord*>(a.records);
  constexpr bool AHEAD = DeltaAheadCfg<T, DK, NW>::FITS, BESIDE = DeltaRevCfg<T, DK, NW>::FITS;
  const auto run = [&](auto kernel) {
    return launch_kernel("delta_rev_scan", kernel, a.G == 1 ? dim3(unsigned(units * parts)) : dim3(unsigned(units * a.G), unsigned(parts)),
                         dim3((AHEAD ? 192 : BESIDE ? 128 : 64) * NW), 0, a.stream, static_cast<const T*>(a.Q), static_cast<const T*>(a.K),
                         static_cast<const T*>(a.dO), a.s, a.seq_len, a.dstate, a.dstate_in, records, a.w_cols, a.zs, a.dstates,
                         a.ends, Divisor(a.H), Divisor(a.G), Divisor(parts), a.seg, a.N, units, a.dv, largest_factor(a.eps));
  };
  if (a.G > 1) {
    hipError_t err;
    if constexpr (AHEAD) err = run(delta_ahead_rev_scan<T, DK, NW, true>);
    else if constexpr (BESIDE) err = run(delta_rev_scan<T, DK, NW, true>);
    else err = run(delta_wide_rev_scan<T, DK, NW, true>);
    if (err == hipSuccess && a.G > 2) err = launch_delta_carry(a, true);
    if (err != hipSuccess) return err;
  }
  if constexpr (AHEAD) return run(delta_ahead_rev_scan<T, DK, NW, false>);
  else if constexpr (BESIDE) return run(delta_rev_scan<T, DK, NW, false>);
  else return run(delta_wide_rev_scan<T, DK, NW, false>);
}

template <typename T, int DK, int DV>
hipError_t run_gradients(const DeltaArgs& a) {
  const int chunks = delta_chunks(a.N);
  return launch_kernel("delta_gradients", delta_gradients<T, DK, DV>, dim3(unsigned(a.B * a.H * chunks)),
                       dim3(DeltaGradCfg<T, DK, DV>::THREADS), 0, a.stream, static_cast<const T*>(a.Q), static_cast<const T*>(a.K),
                       static_cast<const T*>(a.V),
                       static_cast<const T*>(a.dO), a.s, a.log_decay, a.beta, a.seq_len,
                       static_cast<const ChunkRecord*>(a.records), a.errors, a.states, a.zs,
                       a.dstates, static_cast<T*>(a.dQ), static_cast<T*>(a.dK), static_cast<T*>(a.dV), a.dlog_decay, a.dbeta,
                       a.ds_parts, Divisor(a.H), Divisor(chunks), a.N, largest_factor(a.eps), over_eps(a.eps), int(a.state_in != nullptr));
}

template <typename T, int DK>
hipError_t run_backward(const DeltaArgs& a) {
  constexpr int MOST = sizeof(T) == 4 && DK == 128 ? 2 : 4;   // waves that the LDS holds the rows of dO for
  hipError_t err = a.dv == 32 ? run_rev<T, DK, 2>(a) : run_rev<T, DK, MOST>(a);
  if (err != hipSuccess) return err;
  err = a.dv == 32 ? run_gradients<T, DK, 32>(a) : a.dv == 64 ? run_gradients<T, DK, 64>(a) : run_gradients<T, DK, 128>(a);
  if (err != hipSuccess) return err;
  const int units = a.B * a.H, outs = a.seq_len != nullptr ? units : a.H;
  return launch_kernel("delta_sum_ds", delta_sum_ds, dim3(unsigned((outs + 3) / 4)), dim3(256), 0, a.stream, a.ds_parts, a.ds,
                       outs, outs, units, delta_chunks(a.N));
}

}  // namespace

hipError_t DELTA_SYM(delta_bwd)(const DeltaArgs& a) {
  typedef DELTA_T T;
  if (!a.saved) {
    DeltaArgs fwd = a;
    fwd.O = nullptr;
    fwd.state = nullptr;
    const hipError_t err = DELTA_SYM(delta_fwd)(fwd);
    if (err != hipSuccess) return err;
  }
  return a.dk == 32 ? run_backward<T, 32>(a) : a.dk == 64 ? run_backward<T, 64>(a) : run_backward<T, 128>(a);
}

}  // namespace cottn
