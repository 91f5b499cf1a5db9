// Causal cosine attention with a decay for each head, backward (gfx950): the formulas stand in decay.h.  This file builds the
// bfloat16 kernels, the IEEE half ones when it is included with COTTN_ELEM_F16 defined and the fp32 ones with
// COTTN_ELEM_F32 and COTTN_F32_WHOLE.
//
// Two scans of a segment.  The first walks forward in time with H and gives dQ; it also forms G = sum over a chunk's rows of
// g^i' qh_i^T dO_i, from which it leaves the segment's reverse-time total for the second, and ds.  The second walks backward in
// time with R and gives dK and dV.
//
// ds = sum_i (sum_j g^(i-j) (qh_i . kh_j) v_j) . dO_i is a result in fp32 and a sum of terms of both signs, so it is not taken
// from results of rounded operands: the rows before a chunk give g <H, G>, element by element from two fp32 matrices whose
// operands are carried in parts (EXACT_PARTS), and the chunk itself gives the sum of its two masked fp32 tiles' products before
// they are rounded.
//
// The chain rule through x / max(|x|, eps): dx = s r (dxh - xh (xh . dxh)) with r = 1 / max(|x|, eps); rows at or below eps
// have dx = s r dxh.
#include "device_common.h"
#include "launch.h"
#include "tile_io.h"
#include "workspace.h"
#include "decay.h"

namespace cottn {
namespace COTTN_NS {
namespace {

template <int DK, int DV, int C, int CS>
struct DecayBwdCfg {
  static constexpr int RG = C / 16, NW = RG * CS, NT = NW * 64;
  static constexpr int NKT = DK / 16 / CS, NVT = DV / 16 / CS;   // result column tiles of a wave
  static constexpr int KSK = DK / 32, KSV = DV / 32, NP = C / 32;
  static constexpr int TPK = tile_pitch(DK, C), TPV = tile_pitch(DV, C), SP = lds_pitch(DV);
  static constexpr int TILEK = C * TPK, TILEV = C * TPV, STATE = DK * SP;
  static constexpr int LDS_BYTES = LDS_ELEM * (2 * TILEK + 2 * TILEV + STATE) + 4 * 8 * C;
  // dQ rows are staged in the wave's own query rows
  static constexpr int WAVES = decay_waves(LDS_BYTES, NW, CS);
};

// xh . dxh of a row and its removal from dxh, where the tile holds x' with xh = left x'
template <int NTILES>
__device__ __forceinline__ void take_out_row(f32x4* acc, const float (&xv)[NTILES][4], float dot, float left, float whole,
                                             float inv_eps) {
  const float c = whole == inv_eps ? 0.f : left * (left * dot);
#pragma unroll
  for (int nt = 0; nt < NTILES; ++nt)
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[nt][v] -= xv[nt][v] * c;
}

// Factors of rows, which of them by the lane of the row: [0] TILE_UNIT `left`, [1] that times g^e1(row), [2] STATE_UNIT
// left g^e2(row), [3] `whole`.
template <class Stage, int C, class E1, class E2>
__device__ __forceinline__ void store_factors(float* rows, const RowFactors<Stage>& f, const Decay& g, E1 e1, E2 e2) {
  const int which = threadIdx.x % Stage::LPR;
#pragma unroll
  for (int p = 0; p < Stage::PASSES; ++p) {
    const int lr = p * Stage::RPP + threadIdx.x / Stage::LPR;
    const int e = which == 1 ? e1(lr) : which == 2 ? e2(lr) : 0;
    if ((C % Stage::RPP == 0 || lr < C) && which < 4)
      rows[which * C + lr] = (which == 3 ? f.whole[p] : f.left[p]) * g.after(float(e)) *
                             (which == 2 ? STATE_UNIT : which == 3 ? 1.f : TILE_UNIT);
  }
}

// ---------------------------------------------------------------------------------------
// dQ of a segment, first chunk to last.  H and G sit in accumulators with the values down and the keys along, tile (x, y):
// element [v] of lane (r, q4) is H[key 16 col_tile(x) + r][value 16 row_tile(y) + 4 q4 + v].  A wave has few key tiles and all
// values (of its part): fragments of keys and queries are the ones that weights go to, 50 instructions each.  bf16: 96 units
// of 1024 rows 64 x 64 20.9 us (VALU issue 40 %, matrix instructions 16 %); 16 of 65536 rows 155 us, 4.3 TB/s (54 %, 25 %).
template <int DK, int DV, int C, int CS>
COTTN_KERNEL((C * 4 * CS, (DecayBwdCfg<DK, DV, C, CS>::WAVES)), bwd_decay_dq)
    const elem_t* __restrict__ Q, const elem_t* __restrict__ K, const elem_t* __restrict__ V, const elem_t* __restrict__ dO,
    const float* __restrict__ s, const float* __restrict__ log_decay, elem_t* __restrict__ dQ,
    const float* __restrict__ fwd_states, float* __restrict__ rev_totals, float* __restrict__ ds_partial,
    const float* __restrict__ state_in, const int* __restrict__ lengths, Divisor H, Divisor G, int seg_rows, int N, int units,
    float inv_eps, int flags) {
  using Cfg = DecayBwdCfg<DK, DV, C, CS>;
  using ST = AccTiles<DV, DK, Cfg::NW>;   // value rows, key columns
  using StageK = TileStage<DK, C, Cfg::NT>;
  using StageV = TileStage<DV, C, Cfg::NT>;
  constexpr int RG = Cfg::RG, NKT = Cfg::NKT, TPK = Cfg::TPK, TPV = Cfg::TPV, SP = Cfg::SP;
  COTTN_LDS_ARRAY(lds_t, Qs, Cfg::TILEK, 0)
  COTTN_LDS_ARRAY(lds_t, Ks, Cfg::TILEK, 1)
  COTTN_LDS_ARRAY(lds_t, Vs, Cfg::TILEV, 2)
  COTTN_LDS_ARRAY(lds_t, Gs, Cfg::TILEV, 3)
  COTTN_LDS_ARRAY(lds_t, St, Cfg::STATE, 4)
  COTTN_LDS_ARRAY(float, krows, 4 * C, 5)
  COTTN_LDS_ARRAY(float, qrows, 4 * C, 6)
  COTTN_LDS_ARRAY(float, xdot, CS > 1 ? CS * C : 1, 7)
  COTTN_LDS_ARRAY(float, ds_wave, Cfg::NW, 8)
  Unparted un;
  fetch_argument_now(Q, K, V, dO, s, log_decay, dQ, fwd_states, rev_totals, ds_partial, state_in, lengths, H, G, seg_rows, N,
                     units, inv_eps, flags);
  const bool carried = flags & CARRIED;
  int unit, seg;
  unit_and_segment(blockIdx.x, units, G, unit, seg);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int rg = w % RG, cp = w / RG;
  const elem_t* Qu = Q + size_t(unit) * N * DK;
  const elem_t* Ku = K + size_t(unit) * N * DK;
  const elem_t* Vu = V + size_t(unit) * N * DV;
  const elem_t* Gu = dO + size_t(unit) * N * DV;
  elem_t* dQu = dQ + size_t(unit) * N * DK;
  const int there = valid_rows(lengths, unit, H, N), row_begin = seg * seg_rows, piece_end = min(N, row_begin + seg_rows);
  const int row_end = max(row_begin, min(there, piece_end));
  float* ds_out = ds_partial + size_t(unit) * G.n + seg;
  if (row_begin == row_end) {
    if (tid == 0) *ds_out = 0.f;
    zero_rows<DK>(dQu, row_begin, piece_end);
    return;
  }
  StageK qst, kst;
  StageV vst, gst;
  qst.fetch(Qu, row_begin, row_end);
  kst.fetch(Ku, row_begin, row_end);
  vst.fetch(Vu, row_begin, row_end);
  gst.fetch(Gu, row_begin, row_end);
  const int head = unit - quotient(unit, H) * H.n;
  const Decay g(log_decay[head]);
  const float scale = s[lengths != nullptr ? unit : head];

  f32x4 sacc[ST::NCT][ST::NRT], racc[ST::NCT][ST::NRT];
#pragma unroll
  for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
    for (int y = 0; y < ST::NRT; ++y) sacc[x][y] = racc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool active = ST::active(w), with_rev = seg > 0;   // (no workgroup needs the first segment's total)
  if (active && seg > 0) {
    const float* slots = fwd_states + size_t(unit) * G.n * DK * DV;
    add_decayed_states<false>(sacc, carried ? seg : 0, carried ? seg : seg - 1, g, seg_rows, [&](int slot, int x, int y) {
      return *reinterpret_cast<const f32x4*>(slots + size_t(slot) * DK * DV +
                                             tiled_state_offset(ST::col_tile(w, x), ST::row_tile(w, y), DV / 16, l));
    });
  }
  if (active && state_in != nullptr) {
    const float since = STATE_UNIT * g.after(float(row_begin));
    const float* src = state_in + size_t(unit) * DK * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(src + (16 * ST::col_tile(w, x) + r) * DV +
                                                        16 * ST::row_tile(w, y) + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) sacc[x][y][v] = __builtin_fmaf(since, t[v], sacc[x][y][v]);
      }
  }

  const float row = float(16 * rg + r), to_row = TILE_UNIT * g.after(row + 1.f), once = g.after(1.f);
  float on_diagonal[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) on_diagonal[v] = 4 * q4 + v <= r ? g.after(float(r - 4 * q4 - v)) : 0.f;
  const Kept whole_chunk(g, float(C));
  float ds_lane = 0.f;
  RowPieces<DK, NKT> finished;
#pragma unroll
  for (int j = 0; j < RowPieces<DK, NKT>::PER_LANE; ++j) finished.v[j] = uint4{0u, 0u, 0u, 0u};
  const int colk = 16 * NKT * cp;
  for (int row0 = row_begin; row0 < row_end; row0 += C) {
    const int n = min(C, row_end - row0);
    if (active) {
#pragma unroll
      for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
        for (int y = 0; y < ST::NRT; ++y)
          store4_lds(St + (16 * ST::col_tile(w, x) + r) * SP + 16 * ST::row_tile(w, y) + 4 * q4, PER_UNIT * sacc[x][y][0],
                     PER_UNIT * sacc[x][y][1], PER_UNIT * sacc[x][y][2], PER_UNIT * sacc[x][y][3], un);
    }
    {
      RowFactors<StageK> f;
      f.commit(qst, Qs, inv_eps, un);
      store_factors<StageK, C>(qrows, f, g, [](int) { return 0; }, [](int i) { return i; });
      f.commit(kst, Ks, inv_eps, un);
      store_factors<StageK, C>(krows, f, g, [](int j) { return 15 - j % 16; }, [n](int j) { return max(n - 1 - j, 0); });
      vst.commit_plain(Vs, un);
      gst.commit_plain(Gs, un);
    }
    if (row0 + C < row_end) {
      qst.fetch(Qu, row0 + C, row_end);
      kst.fetch(Ku, row0 + C, row_end);
      vst.fetch(Vu, row0 + C, row_end);
      gst.fetch(Gu, row0 + C, row_end);
    }
    if (row0 > row_begin) store_row_pieces<DK, NKT>(finished, dQu, row0 - C + 16 * rg, row_end, l, colk);
    __syncthreads();

    // G of the chunk, ds of the rows before it, and the segment's reverse-time total, a few value tiles at a time
    if (active) {
      const WeightedTile<ST, Cfg::NP, TPK, EXACT_PARTS> q(Qs, qrows + 2 * C, w, r, q4);
      const float at = g.after(float(row0 - row_begin));
      constexpr int YN = ST::NRT < 4 ? ST::NRT : 4;
      float t = 0.f;
#pragma unroll
      for (int y0 = 0; y0 < ST::NRT; y0 += YN) {
        f32x4 gacc[ST::NCT][YN];
#pragma unroll
        for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
          for (int y = 0; y < YN; ++y) gacc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
        q.template add<YN, TPV>(Gs, y0, w, r, q4, [&](int x, int y) -> f32x4& { return gacc[x][y]; });
#pragma unroll
        for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
          for (int y = 0; y < YN; ++y)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              t = __builtin_fmaf(sacc[x][y0 + y][v], gacc[x][y][v], t);
              racc[x][y0 + y][v] = __builtin_fmaf(at, gacc[x][y][v], racc[x][y0 + y][v]);
            }
      }
      ds_lane += PER_UNIT * PER_UNIT * once * t;
    }

    // what the state gives: dqh^T = H dO^T, then the row's factor
    frag8 gf[Cfg::KSV], qf[Cfg::KSK];
#pragma unroll
    for (int ks = 0; ks < Cfg::KSV; ++ks) gf[ks] = lds_row_frag(Gs + (16 * rg + r) * TPV + 32 * ks, q4);
#pragma unroll
    for (int ks = 0; ks < Cfg::KSK; ++ks) qf[ks] = lds_row_frag(Qs + (16 * rg + r) * TPK + 32 * ks, q4);
    f32x4 dq[NKT];
#pragma unroll
    for (int nt = 0; nt < NKT; ++nt) dq[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < Cfg::KSV; ++ks) {
      frag8 sf[NKT];
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) sf[nt] = lds_row_frag(St + (colk + 16 * nt + r) * SP + 32 * ks, q4);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) dq[nt] = mma16(sf[nt], gf[ks], dq[nt]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int nt = 0; nt < NKT; ++nt)
#pragma unroll
      for (int v = 0; v < 4; ++v) dq[nt][v] *= to_row;

    // the chunk itself, 32 tokens at a time
    float ds_row = 0.f;
#pragma unroll
    for (int p = 0; p < Cfg::NP; ++p) {
      if (2 * p > rg) break;   // wave-uniform: every key is masked from here on
      const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
      f32x4 ta[2], tp[2];
      {
        frag8 vr[2][Cfg::KSV];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSV; ++ks) vr[half][ks] = lds_row_frag(Vs + (16 * (2 * p + half) + r) * TPV + 32 * ks, q4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          ta[half] = tp[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < Cfg::KSV; ++ks) ta[half] = mma16(vr[half][ks], gf[ks], ta[half]);
        }
      }
      if (CS == 1 || cp == p % CS) {   // (one wave of a row group forms the tiles of ds)
        frag8 kr[2][Cfg::KSK];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) kr[half][ks] = lds_row_frag(Ks + (16 * (2 * p + half) + r) * TPK + 32 * ks, q4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) tp[half] = mma16(kr[half][ks], qf[ks], tp[half]);
      }
      frag8 kc[NKT], af;
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) kc[nt] = lds_col_frag(Ks, TPK, t0, t1, colk + 16 * nt, r);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int jt = 2 * p + half;
        // ta[half][v] = dO_(16 rg + r) . v_(16 jt + 4 q4 + v)
        const f32x4 kj = *reinterpret_cast<const f32x4*>(krows + (jt == rg ? 0 : C) + 16 * jt + 4 * q4);
        const float below = g.after(row - float(16 * jt + 15));   // (jt < rg)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          ta[half][v] = jt > rg ? 0.f : ta[half][v] * (kj[v] * (jt == rg ? on_diagonal[v] : below));
          ds_row = __builtin_fmaf(tp[half][v], ta[half][v], ds_row);
        }
        put_four(af, half, ta[half]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) dq[nt] = mma16_add(kc[nt], af, dq[nt]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the state after the chunk, but for the last (with the same in the other scans, 96 units of 1024 rows 64 x 64 63.7 -> 62.0
    // us, 128 x 128 156.6 -> 155.2 where this scan forms it all the same and 157.9 where not)
    if (active && ((DK == 128 && DV == 128) || row0 + C < row_end)) {
      (n == C ? whole_chunk : Kept(g, float(n))).on(sacc);   // (the gradients of a state with an infinite element are not finite)
      const WeightedTile<ST, Cfg::NP, TPK, EXACT_PARTS> k(Ks, krows + 2 * C, w, r, q4);
      constexpr int YN = ST::NRT < 4 ? ST::NRT : 4;
#pragma unroll
      for (int y0 = 0; y0 < ST::NRT; y0 += YN)
        k.template add<YN, TPV>(Vs, y0, w, r, q4, [&](int x, int y) -> f32x4& { return sacc[x][y0 + y]; });
    }

    const float left = 1.f / TILE_UNIT * qrows[16 * rg + r], whole = qrows[3 * C + 16 * rg + r];
    ds_lane += 1.f / TILE_UNIT * left * ds_row;
    float xv[NKT][4];
    float t = dot_with_row<NKT, TPK>(dq, Qs + 16 * rg * TPK, colk, xv, r, q4);
    if (CS > 1) {   // the row's dot product over the columns of all its waves
      if (q4 == 0) xdot[cp * C + 16 * rg + r] = t;
      __syncthreads();
      t = 0.f;
#pragma unroll
      for (int i = 0; i < CS; ++i) t += xdot[i * C + 16 * rg + r];
    }
    take_out_row<NKT>(dq, xv, t, left, whole, inv_eps);
    // every wave has read all query rows for G: they take the finished ones
    if (CS == 1) __syncthreads();
    gather_rows_transposed<DK, NKT>(dq, 1.f / TILE_UNIT * scale * whole, Qs + 16 * rg * TPK, l, finished, un, colk);
    __syncthreads();
  }
  store_row_pieces<DK, NKT>(finished, dQu, row_begin + (row_end - row_begin - 1) / C * C + 16 * rg, row_end, l, colk);
  if (lengths != nullptr) zero_rows<DK>(dQu, row_end, piece_end);
  if (with_rev && active) {
    float* out = rev_totals + (size_t(unit) * G.n + seg) * DK * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y)
        store_state_words(out + tiled_state_offset(ST::col_tile(w, x), ST::row_tile(w, y), DV / 16, l), racc[x][y]);
  }
  ds_lane = group_sum<64>(ds_lane);
  if (l == 0) ds_wave[w] = ds_lane;
  __syncthreads();
  if (tid == 0) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < Cfg::NW; ++i) t += ds_wave[i];
    *ds_out = t;
  }
}

// ---------------------------------------------------------------------------------------
// dK and dV of a segment, last chunk to first.  R sits in accumulators with the values down and the keys along, tile (x, y):
// element [v] of lane (r, q4) is R[key 16 col_tile(x) + r][value 16 row_tile(y) + 4 q4 + v].  The first workgroups also add up
// ds from what the dQ scan left.  PARTS: EXACT_PARTS where the reverse-time state is asked for.  bf16: 96 units of 1024 rows
// 64 x 64 18.5 us (VALU issue 34 %, matrix instructions 13 %, LDS 37 %); 16 of 65536 rows 151 us, 5.3 TB/s.
template <int DK, int DV, int C, int CS, int PARTS>
COTTN_KERNEL((C * 4 * CS, (DecayBwdCfg<DK, DV, C, CS>::WAVES)), bwd_decay_dkdv)
    const elem_t* __restrict__ Q, const elem_t* __restrict__ K, const elem_t* __restrict__ V, const elem_t* __restrict__ dO,
    const float* __restrict__ s, const float* __restrict__ log_decay, elem_t* __restrict__ dK, elem_t* __restrict__ dV,
    const float* __restrict__ rev_states, const float* __restrict__ ds_partial, float* __restrict__ ds,
    const float* __restrict__ rev_in, float* __restrict__ rev_out, const int* __restrict__ lengths, int B, Divisor H, Divisor G,
    int seg_rows, int N, float inv_eps, int flags) {
  using Cfg = DecayBwdCfg<DK, DV, C, CS>;
  using ST = AccTiles<DV, DK, Cfg::NW>;   // value rows, key columns
  using StageK = TileStage<DK, C, Cfg::NT>;
  using StageV = TileStage<DV, C, Cfg::NT>;
  constexpr int RG = Cfg::RG, NKT = Cfg::NKT, NVT = Cfg::NVT, TPK = Cfg::TPK, TPV = Cfg::TPV, SP = Cfg::SP;
  COTTN_LDS_ARRAY(lds_t, Qs, Cfg::TILEK, 0)
  COTTN_LDS_ARRAY(lds_t, Ks, Cfg::TILEK, 1)
  COTTN_LDS_ARRAY(lds_t, Vs, Cfg::TILEV, 2)
  COTTN_LDS_ARRAY(lds_t, Gs, Cfg::TILEV, 3)
  COTTN_LDS_ARRAY(lds_t, Rl, Cfg::STATE, 4)
  COTTN_LDS_ARRAY(float, krows, 4 * C, 5)
  COTTN_LDS_ARRAY(float, qrows, 4 * C, 6)
  COTTN_LDS_ARRAY(float, xdot, CS > 1 ? CS * C : 1, 7)
  Unparted un;
  fetch_argument_now(Q, K, V, dO, s, log_decay, dK, dV, rev_states, ds_partial, ds, rev_in, rev_out, lengths, B, H, G, seg_rows,
                     N, inv_eps, flags);
  const bool carried = flags & CARRIED, stream = flags & STREAM;
  int unit, seg;
  unit_and_segment(blockIdx.x, B * H.n, G, unit, seg);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int rg = w % RG, cp = w / RG;
  const elem_t* Qu = Q + size_t(unit) * N * DK;
  const elem_t* Ku = K + size_t(unit) * N * DK;
  const elem_t* Vu = V + size_t(unit) * N * DV;
  const elem_t* Gu = dO + size_t(unit) * N * DV;
  elem_t* dKu = dK + size_t(unit) * N * DK;
  elem_t* dVu = dV + size_t(unit) * N * DV;
  const int there = valid_rows(lengths, unit, H, N), row_begin = seg * seg_rows, piece_end = min(N, row_begin + seg_rows);
  const int row_end = max(row_begin, min(there, piece_end));
  const int last_row0 = row_begin + (row_end - row_begin - 1) / C * C;
  StageK qst, kst;
  StageV vst, gst;
  if (row_begin < row_end) {
    qst.fetch(Qu, last_row0, row_end, stream);
    kst.fetch(Ku, last_row0, row_end, stream);
    vst.fetch(Vu, last_row0, row_end, stream);
    gst.fetch(Gu, last_row0, row_end, stream);
  }
  // ds[h]: over batches and segments; with lengths ds[b][h], over segments
  if (int(blockIdx.x) < (lengths != nullptr ? B * H.n : H.n) && w == 0) {
    float t = 0.f;
    const int n = lengths != nullptr ? G.n : B * G.n;
    for (int i = l; i < n; i += 64)
      t += lengths != nullptr ? ds_partial[size_t(blockIdx.x) * G.n + i]
                              : ds_partial[(size_t(quotient(i, G)) * H.n + blockIdx.x) * G.n + (i - quotient(i, G) * G.n)];
    t = group_sum<64>(t);
    if (l == 0) ds[blockIdx.x] = t;
  }
  if (row_begin == row_end && seg > 0) {
    zero_rows<DK>(dKu, row_begin, piece_end);
    zero_rows<DV>(dVu, row_begin, piece_end);
    return;
  }
  const int head = unit - quotient(unit, H) * H.n;
  const Decay g(log_decay[head]);
  const float scale = s[lengths != nullptr ? unit : head];

  f32x4 racc[ST::NCT][ST::NRT];
#pragma unroll
  for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
    for (int y = 0; y < ST::NRT; ++y) racc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool active = ST::active(w);
  if (active && there > piece_end) {
    const float* slots = rev_states + size_t(unit) * G.n * DK * DV;
    const int last = (there - 1) / seg_rows;
    add_decayed_states<true>(racc, carried ? seg : seg + 1, carried ? seg : last, g, seg_rows, [&](int slot, int x, int y) {
      return *reinterpret_cast<const f32x4*>(slots + size_t(slot) * DK * DV +
                                             tiled_state_offset(ST::col_tile(w, x), ST::row_tile(w, y), DV / 16, l));
    });
  }
  bool infinite = false;
  if (active && rev_in != nullptr) {
    const float until = STATE_UNIT * g.after(float(there - row_end));
    const float* src = rev_in + size_t(unit) * DK * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(src + (16 * ST::col_tile(w, x) + r) * DV +
                                                        16 * ST::row_tile(w, y) + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) racc[x][y][v] = __builtin_fmaf(until, t[v], racc[x][y][v]);
      }
    infinite = any_infinite(racc);
  }

  const float row = float(16 * rg + r);   // of the chunk: this lane's key
  float on_diagonal[4];                   // g^(i-j) for the queries i of the tile of the wave's own rows
#pragma unroll
  for (int v = 0; v < 4; ++v) on_diagonal[v] = 4 * q4 + v >= r ? g.after(float(4 * q4 + v - r)) : 0.f;
  const Kept whole_chunk(g, float(C));
  const int colk = 16 * NKT * cp, colv = 16 * NVT * cp;
  RowPieces<DK, NKT> done_k;
  RowPieces<DV, NVT> done_v;
#pragma unroll
  for (int j = 0; j < RowPieces<DK, NKT>::PER_LANE; ++j) done_k.v[j] = uint4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < RowPieces<DV, NVT>::PER_LANE; ++j) done_v.v[j] = uint4{0u, 0u, 0u, 0u};
  for (int row0 = last_row0; row0 >= row_begin && row_begin < row_end; row0 -= C) {
    const int n = min(C, row_end - row0);
    if (active) {
#pragma unroll
      for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
        for (int y = 0; y < ST::NRT; ++y)
          store4_lds(Rl + (16 * ST::col_tile(w, x) + r) * SP + 16 * ST::row_tile(w, y) + 4 * q4, PER_UNIT * racc[x][y][0],
                     PER_UNIT * racc[x][y][1], PER_UNIT * racc[x][y][2], PER_UNIT * racc[x][y][3], un);
      (n == C ? whole_chunk : Kept(g, float(n))).on(racc, infinite);
    }
    {
      RowFactors<StageK> f;
      f.commit(qst, Qs, inv_eps, un);
      store_factors<StageK, C>(qrows, f, g, [](int i) { return i % 16; }, [](int i) { return i; });
      f.commit(kst, Ks, inv_eps, un);
      store_factors<StageK, C>(krows, f, g, [](int) { return 0; }, [](int) { return 0; });
      vst.commit_plain(Vs, un);
      gst.commit_plain(Gs, un);
    }
    if (row0 > row_begin) {
      qst.fetch(Qu, row0 - C, row_end, stream);
      kst.fetch(Ku, row0 - C, row_end, stream);
      vst.fetch(Vu, row0 - C, row_end, stream);
      gst.fetch(Gu, row0 - C, row_end, stream);
    }
    if (row0 < last_row0) {
      store_row_pieces<DK, NKT>(done_k, dKu, row0 + C + 16 * rg, row_end, l, colk);
      store_row_pieces<DV, NVT>(done_v, dVu, row0 + C + 16 * rg, row_end, l, colv);
    }
    __syncthreads();

    // what the state gives: dv^T = R^T k^T and dkh^T = R v^T, then the rows' factors
    frag8 kf[Cfg::KSK], vf[Cfg::KSV];
#pragma unroll
    for (int ks = 0; ks < Cfg::KSK; ++ks) kf[ks] = lds_row_frag(Ks + (16 * rg + r) * TPK + 32 * ks, q4);
#pragma unroll
    for (int ks = 0; ks < Cfg::KSV; ++ks) vf[ks] = lds_row_frag(Vs + (16 * rg + r) * TPV + 32 * ks, q4);
    const float left = 1.f / TILE_UNIT * krows[16 * rg + r], whole = krows[3 * C + 16 * rg + r];
    f32x4 dk[NKT], dv[NVT];
#pragma unroll
    for (int nt = 0; nt < NKT; ++nt) dk[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nt = 0; nt < NVT; ++nt) dv[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < Cfg::KSK; ++ks) {
      frag8 rcol[NVT];
#pragma unroll
      for (int nt = 0; nt < NVT; ++nt) rcol[nt] = lds_col_frag_ks(Rl, SP, ks, q4, colv + 16 * nt, r);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NVT; ++nt) dv[nt] = mma16(rcol[nt], kf[ks], dv[nt]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int ks = 0; ks < Cfg::KSV; ++ks) {
      frag8 rrow[NKT];
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) rrow[nt] = lds_row_frag(Rl + (colk + 16 * nt + r) * SP + 32 * ks, q4);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) dk[nt] = mma16(rrow[nt], vf[ks], dk[nt]);
      __builtin_amdgcn_sched_barrier(0);
    }
    const float to_end = g.after(fmaxf(float(n) - row, 0.f));
#pragma unroll
    for (int nt = 0; nt < NVT; ++nt)
#pragma unroll
      for (int v = 0; v < 4; ++v) dv[nt][v] *= left * to_end;
#pragma unroll
    for (int nt = 0; nt < NKT; ++nt)
#pragma unroll
      for (int v = 0; v < 4; ++v) dk[nt][v] *= TILE_UNIT * to_end;

    // the chunk itself, 32 queries at a time
#pragma unroll
    for (int p = 0; p < Cfg::NP; ++p) {
      if (2 * p + 1 < rg) continue;   // wave-uniform: every query is masked
      const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
      f32x4 tp[2], ta[2];
      {
        frag8 qr[2][Cfg::KSK];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) qr[half][ks] = lds_row_frag(Qs + (16 * (2 * p + half) + r) * TPK + 32 * ks, q4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          tp[half] = ta[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) tp[half] = mma16(qr[half][ks], kf[ks], tp[half]);
        }
      }
      {
        frag8 gr[2][Cfg::KSV];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSV; ++ks) gr[half][ks] = lds_row_frag(Gs + (16 * (2 * p + half) + r) * TPV + 32 * ks, q4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSV; ++ks) ta[half] = mma16(gr[half][ks], vf[ks], ta[half]);
      }
      frag8 pf, af, gc[NVT], qc[NKT];
#pragma unroll
      for (int nt = 0; nt < NVT; ++nt) gc[nt] = lds_col_frag(Gs, TPV, t0, t1, colv + 16 * nt, r);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int it = 2 * p + half;
        // tp[half][v] = q_(16 it + 4 q4 + v) . k_(16 rg + r), a row's factor at a time (decay.h: RowFactors)
        const f32x4 qi = *reinterpret_cast<const f32x4*>(qrows + (it == rg ? 0 : C) + 16 * it + 4 * q4);
        const float above = g.after(float(16 * it) - row);   // (it > rg)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float f = it < rg ? 0.f : qi[v] * (it == rg ? on_diagonal[v] : above);
          tp[half][v] = it < rg ? 0.f : tp[half][v] * f * (1.f / TILE_UNIT * left);
          ta[half][v] = it < rg ? 0.f : ta[half][v] * f;
        }
        put_four(pf, half, tp[half]);
        put_four(af, half, ta[half]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NVT; ++nt) dv[nt] = mma16_add(gc[nt], pf, dv[nt]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) qc[nt] = lds_col_frag(Qs, TPK, t0, t1, colk + 16 * nt, r);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nt = 0; nt < NKT; ++nt) dk[nt] = mma16_add(qc[nt], af, dk[nt]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the state before the chunk, if somebody takes it
    if (active && (row0 > row_begin || (rev_out != nullptr && seg == 0))) {
      const WeightedTile<ST, Cfg::NP, TPK, PARTS> q(Qs, qrows + 2 * C, w, r, q4);
      constexpr int YN = ST::NRT < 4 ? ST::NRT : 4;
#pragma unroll
      for (int y0 = 0; y0 < ST::NRT; y0 += YN)
        q.template add<YN, TPV>(Gs, y0, w, r, q4, [&](int x, int y) -> f32x4& { return racc[x][y0 + y]; });
    }

    float xv[NKT][4];
    float t = dot_with_row<NKT, TPK>(dk, Ks + 16 * rg * TPK, colk, xv, r, q4);
    if (CS > 1) {
      if (q4 == 0) xdot[cp * C + 16 * rg + r] = t;
      __syncthreads();   // and the rows of Ks and Vs are read by all waves of the row group
      t = 0.f;
#pragma unroll
      for (int i = 0; i < CS; ++i) t += xdot[i * C + 16 * rg + r];
    }
    take_out_row<NKT>(dk, xv, t, left, whole, inv_eps);
    // (the row group's own rows of Ks and Vs are read by its own waves only)
    if (CS == 1) wave_lds_sync();
    gather_rows_transposed<DK, NKT>(dk, 1.f / TILE_UNIT * scale * whole, Ks + 16 * rg * TPK, l, done_k, un, colk);
    gather_rows_transposed<DV, NVT>(dv, scale, Vs + 16 * rg * TPV, l, done_v, un, colv);
    __syncthreads();
  }
  if (row_begin < row_end) {
    store_row_pieces<DK, NKT>(done_k, dKu, row_begin + 16 * rg, row_end, l, colk);
    store_row_pieces<DV, NVT>(done_v, dVu, row_begin + 16 * rg, row_end, l, colv);
  }
  if (lengths != nullptr) {
    zero_rows<DK>(dKu, row_end, piece_end);
    zero_rows<DV>(dVu, row_end, piece_end);
  }
  if (rev_out != nullptr && seg == 0 && active) {
    float* out = rev_out + size_t(unit) * DK * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y)
        *reinterpret_cast<f32x4*>(out + (16 * ST::col_tile(w, x) + r) * DV + 16 * ST::row_tile(w, y) + 4 * q4) =
            PER_UNIT * racc[x][y];
  }
}

template <int DK, int DV, int C, int CS>
hipError_t run_bwd_decay(const DecayArgs& a) {
  const int units = a.B * a.H;
  const elem_t* Q = static_cast<const elem_t*>(a.Q);
  const elem_t* K = static_cast<const elem_t*>(a.K);
  const elem_t* V = static_cast<const elem_t*>(a.V);
  const elem_t* dO = static_cast<const elem_t*>(a.dO);
  char* ws = static_cast<char*>(a.workspace);
  const size_t states = state_slots_bytes(a.G > 1 ? long(units) * a.G : 0, DK, DV);
  float* own_fwd = reinterpret_cast<float*>(ws);
  float* rev = reinterpret_cast<float*>(ws + states);
  float* ds_partial = reinterpret_cast<float*>(ws + 2 * states);
  const float* fwd = a.saved_fwd_states;
  hipError_t err = hipSuccess;
  if (a.G > 1 && fwd == nullptr) {
    err = COTTN_SYM(launch_decay_totals)(a, own_fwd);
    if (err == hipSuccess && a.carried) err = launch_decay_carry(a, own_fwd, false);
    if (err != hipSuccess) return err;
    fwd = own_fwd;
  }
  // The second scan is the last to read the rows: past the caches where they hold no call's tensors (768 units of 512 rows 128
  // x 128, forward + backward 436 -> 419 us, 16 of 65536 rows 64 x 64 488 -> 473; where they do, 96 of 1024 rows, 63.7 -> 64.8;
  // and the first scan too, 426 and 478).
  const double bytes = 2.0 * units * double(a.N) * (DK + DV) * ELEM;
  const int flags = (a.carried ? CARRIED : 0) | (bytes > 256.0 * 1024 * 1024 ? STREAM : 0);
  const dim3 grid(units * a.G), block(64 * (C / 16) * CS);
  const Divisor H(a.H), G(a.G);
  const float inv_eps = 1.0f / a.eps;
  err = launch_kernel(COTTN_SYM_STR(bwd_decay_dq), COTTN_SYM(bwd_decay_dq)<DK, DV, C, CS>, grid, block, 0, a.stream, Q, K, V, dO, a.s,
                      a.log_decay, static_cast<elem_t*>(a.dQ), fwd, rev, ds_partial, a.state_in, a.seq_len, H, G, a.seg_rows, a.N,
                      units, inv_eps, flags);
  if (err == hipSuccess && a.G > 1 && a.carried) err = launch_decay_carry(a, rev, true);
  if (err != hipSuccess) return err;
  const auto dkdv = [&](auto kernel) {
    return launch_kernel(COTTN_SYM_STR(bwd_decay_dkdv), kernel, grid, block, 0, a.stream, Q, K, V, dO, a.s, a.log_decay,
                         static_cast<elem_t*>(a.dK), static_cast<elem_t*>(a.dV), rev, ds_partial, a.ds, a.rev_state_in,
                         a.rev_state_out, a.seq_len, a.B, H, G, a.seg_rows, a.N, inv_eps, flags);
  };
  if (a.rev_state_out != nullptr) return dkdv(COTTN_SYM(bwd_decay_dkdv)<DK, DV, C, CS, EXACT_PARTS>);
  return dkdv(COTTN_SYM(bwd_decay_dkdv)<DK, DV, C, CS, ROUNDED_PARTS>);
}

}  // namespace
}  // namespace COTTN_NS

using namespace COTTN_NS;

// Rows of a chunk and waves on a row group, as in the backward without decay (bwd_causal_bf16.hip: BwdSplit).  96 units of 1024
// rows, forward + backward, bf16: 64 x 64 one wave / two 63.5 / 103 us, 128 x 128 64 rows / 32 157 / 250, 128 x 64 32 rows / 64
// rows, each with two waves, 106 / 264: the others do not fit their registers.  fp32 384 units of 512 rows, two waves / four:
// 128 x 64 635 / 629, 64 x 128 579 / 596.
hipError_t COTTN_SYM(bwd_decay)(const DecayArgs& a) {
#define COTTN_CASE(DK, DV)                                                                                             \
  case DK * 1000 + DV: {                                                                                               \
    constexpr bool WIDE = DK != DV && DK >= 64 && DV >= 64;                                                            \
    return run_bwd_decay<DK, DV, ELEM_IS_F32 || WIDE ? 32 : 64, ELEM_IS_F32 || WIDE || (DK == 128 && DV == 128) ? 2 : 1>(a); \
  }
  switch (a.dk * 1000 + a.dv) {
    COTTN_CASE(32, 32) COTTN_CASE(32, 64) COTTN_CASE(32, 128) COTTN_CASE(64, 32) COTTN_CASE(64, 64) COTTN_CASE(64, 128)
    COTTN_CASE(128, 32) COTTN_CASE(128, 64) COTTN_CASE(128, 128)
    default: return hipErrorInvalidValue;
  }
#undef COTTN_CASE
}

}  // namespace cottn
