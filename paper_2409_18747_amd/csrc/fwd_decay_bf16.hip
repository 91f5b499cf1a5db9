// Causal cosine attention with a decay for each head, forward (gfx950): the formulas stand in decay.h.  This file builds the
// bfloat16 kernels, the IEEE half ones when it is included with COTTN_ELEM_F16 defined and the fp32 ones with
// COTTN_ELEM_F32 and COTTN_F32_WHOLE.
//
// A workgroup walks a segment of a (batch, head) chunk by chunk with the d_key x d_value state in fp32 accumulators.  Of a
// chunk it forms the masked tiles (Qh Kh^T (.) g^(i-j)) and their product with V, adds what the state gives, and takes the
// state on to the chunk's end.  Where a sequence is cut into segments, a first kernel leaves the total of every segment but the
// last, each as seen from the segment's own end; the scans weigh and add those before theirs.
//
// What bounds them: vector instructions (the weights of operand fragments, their parts, the masked tiles) and the rows' way
// through memory, at some 4 to 5.4 TB/s for large calls; matrix instructions take a quarter of the time.
#include "device_common.h"
#include "launch.h"
#include "tile_io.h"
#include "decay.h"

namespace cottn {
namespace COTTN_NS {
namespace {

template <int DK, int DV, int C, int CS>
struct DecayFwdCfg {
  static constexpr int RG = C / 16, NW = RG * CS, NT = NW * 64;   // row groups, waves, threads
  static constexpr int KSK = DK / 32, NP = C / 32, NOT = DV / 16 / CS;
  static constexpr int TPK = tile_pitch(DK, C), TPV = tile_pitch(DV, C), SP = lds_pitch(DV);
  static constexpr int TILEK = C * TPK, TILEV = C * TPV, STATE = DK * SP;
  // finished rows are staged in the wave's own query rows where nobody else reads those and they are wide enough
  static constexpr bool OWN_STAGE = CS > 1 || ELEM * stage_pitch(DV) > LDS_ELEM * TPK;
  static constexpr int OP = stage_tile_pitch(DV, C);
  static constexpr int LDS_BYTES = LDS_ELEM * (2 * TILEK + TILEV + STATE) + (OWN_STAGE ? ELEM * C * OP : 0) + 4 * 4 * C;
  static constexpr int WAVES = decay_waves(LDS_BYTES, NW, CS);
};

// In either kernel a wave holds tiles of the state with the values down and the keys along: element [v] of lane (r, q4) of tile
// (x, y) is S[key 16 col_tile(x) + r][value 16 row_tile(y) + 4 q4 + v].  It has few key tiles and as many values as that
// leaves: the fragments of keys are the ones that weights go to, some 50 instructions each.

// The factors of the chunk's key rows, one lane of a row for each: [0] 1 / norm, [1] that times g^(15 - j' mod 16), for tiles
// below the diagonal, [2] times g^(n-1-j') STATE_UNIT, for the state after the chunk's n rows.
template <class Stage, int C>
__device__ __forceinline__ void store_key_factors(float* rows, const RowFactors<Stage>& f, const Decay& g, int n) {
  const int which = threadIdx.x % Stage::LPR;
#pragma unroll
  for (int p = 0; p < Stage::PASSES; ++p) {
    const int lr = p * Stage::RPP + threadIdx.x / Stage::LPR;
    const int e = which == 0 ? 0 : which == 1 ? 15 - lr % 16 : max(n - 1 - lr, 0);
    if ((C % Stage::RPP == 0 || lr < C) && which < 3)
      rows[which * C + lr] = f.left[p] * g.after(float(e)) * (which == 2 ? STATE_UNIT : 1.f);
  }
}

// ---------------------------------------------------------------------------------------
// T[unit][segment] = sum over the rows j of a segment of g^(end-1-j) kh_j^T v_j, for all segments but the last of a unit (and
// those that a sequence of a padded batch does not reach), as tiles in accumulator order.  96 units of 1024 rows 64 x 64 in
// bf16, 4 segments, 8.8 us; 16 of 65536 rows, 32 segments, 55.8 us, 4.8 TB/s (VALU issue 57 %, matrix instructions 21 %).
template <int DK, int DV, int C>
COTTN_KERNEL((C * 4), decay_segment_state)
    const elem_t* __restrict__ K, const elem_t* __restrict__ V, float* __restrict__ seg_state,
    const float* __restrict__ log_decay, const int* __restrict__ lengths, Divisor H, Divisor G, int seg_rows, int N,
    int units, float inv_eps) {
  using Cfg = DecayFwdCfg<DK, DV, C, 1>;
  using ST = AccTiles<DV, DK, Cfg::NW>;
  using StageK = TileStage<DK, C, Cfg::NT>;
  using StageV = TileStage<DV, C, Cfg::NT>;
  COTTN_LDS_ARRAY(lds_t, Ks, Cfg::TILEK, 0)
  COTTN_LDS_ARRAY(lds_t, Vs, Cfg::TILEV, 1)
  COTTN_LDS_ARRAY(float, rows, 3 * C, 2)
  Unparted un;
  fetch_argument_now(K, V, seg_state, log_decay, lengths, H, G, seg_rows, N, units, inv_eps);
  int unit, seg;
  unit_and_segment(blockIdx.x, units, G, unit, seg);
  if (seg == G.n - 1) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const elem_t* Ku = K + size_t(unit) * N * DK;
  const elem_t* Vu = V + size_t(unit) * N * DV;
  const int row_begin = seg * seg_rows, row_end = min(valid_rows(lengths, unit, H, N), row_begin + seg_rows);
  StageK kst;
  StageV vst;
  kst.fetch(Ku, row_begin, row_end);
  vst.fetch(Vu, row_begin, row_end);
  const Decay g(log_decay[unit - quotient(unit, H) * H.n]);
  const Kept whole_chunk(g, float(C));
  f32x4 acc[ST::NCT][ST::NRT];
#pragma unroll
  for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
    for (int y = 0; y < ST::NRT; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int row0 = row_begin; row0 < row_end; row0 += C) {
    __syncthreads();   // the reads of the chunk before are done
    RowFactors<StageK> kf;
    kf.commit(kst, Ks, inv_eps, un);
    const int n = min(C, row_end - row0);   // (fp32 segments are whole chunks of 32 rows, not of this kernel's 64)
    store_key_factors<StageK, C>(rows, kf, g, n);
    vst.commit_plain(Vs, un);
    if (row0 + C < row_end) {
      kst.fetch(Ku, row0 + C, row_end);
      vst.fetch(Vu, row0 + C, row_end);
    }
    __syncthreads();
    if (ST::active(w)) {
      (n == C ? whole_chunk : Kept(g, float(n))).on(acc);
      const WeightedTile<ST, Cfg::NP, Cfg::TPK, EXACT_PARTS> k(Ks, rows + 2 * C, w, r, q4);
      constexpr int YN = ST::NRT < 4 ? ST::NRT : 4;
#pragma unroll
      for (int y0 = 0; y0 < ST::NRT; y0 += YN)
        k.template add<YN, Cfg::TPV>(Vs, y0, w, r, q4, [&](int x, int y) -> f32x4& { return acc[x][y0 + y]; });
    }
  }
  if (ST::active(w)) {
    float* out = seg_state + (size_t(unit) * G.n + seg) * DK * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y)
        store_state_words(out + tiled_state_offset(ST::col_tile(w, x), ST::row_tile(w, y), DV / 16, l), acc[x][y]);
  }
}

// ---------------------------------------------------------------------------------------
// Row parts: the chunks of a sequence of one segment, dealt to workgroups that each form the state up to theirs by themselves.
// A chunk that only makes the state takes about half the time of a whole one, so part k takes `most` chunks less half of those
// before it.
__device__ __forceinline__ void row_part(int k, int most, int& begin, int& count) {
  begin = 0;
  count = most;
  for (int i = 0; i < k; ++i) {
    begin += count;
    count = max(1, most - begin / 2);
  }
}

// The scan of one segment.  Wave (row group rg, column part cp) owns the query rows 16 rg .. of the chunk and the output
// columns of its part, and tiles of the state, held as said above.  Results are accumulated transposed: a lane holds four
// consecutive columns of one output row.  LDV > DV (one segment): a workgroup takes DV of the LDV value columns, which the
// whole computation leaves apart from one another but for the masked tiles, formed LDV / DV times, and a part of the rows
// (row_part). PARTS: EXACT_PARTS where the state is asked for.
//   bf16: 96 units of 1024 rows 64 x 64 in 4 segments 14.4 us; 16 of 65536 rows in 32 segments 99 us, 5.4 TB/s; 1024 of 2048
// rows 128 x 128 558 us, 3.8 TB/s (VALU issue 47 %, matrix instructions 28 %, LDS 46 % of the time).
template <int DK, int DV, int C, int CS, int PARTS, int LDV = DV>
COTTN_KERNEL((C * 4 * CS, (DecayFwdCfg<DK, DV, C, CS>::WAVES)), fwd_decay_scan)
    const elem_t* __restrict__ Q, const elem_t* __restrict__ K, const elem_t* __restrict__ V,
    const float* __restrict__ s, const float* __restrict__ log_decay, elem_t* __restrict__ O,
    float* __restrict__ state_out, const float* __restrict__ seg_states, const float* __restrict__ state_in,
    const int* __restrict__ lengths, Divisor H, Divisor G, int seg_rows, int N, int units, float inv_eps, int flags) {
  using Cfg = DecayFwdCfg<DK, DV, C, CS>;
  using ST = AccTiles<DV, DK, Cfg::NW>;   // value rows, key columns
  using StageK = TileStage<DK, C, Cfg::NT>;
  using StageV = TileStage<DV, C, Cfg::NT, LDV>;
  constexpr int RG = Cfg::RG, NOT = Cfg::NOT, TPK = Cfg::TPK, TPV = Cfg::TPV, SP = Cfg::SP;
  COTTN_LDS_ARRAY(lds_t, Qs, Cfg::TILEK, 0)
  COTTN_LDS_ARRAY(lds_t, Ks, Cfg::TILEK, 1)
  COTTN_LDS_ARRAY(lds_t, Vs, Cfg::TILEV, 2)
  COTTN_LDS_ARRAY(lds_t, Sl, Cfg::STATE, 3)   // the state, [d_key][d_value], rounded to the element type
  COTTN_LDS_ARRAY(elem_t, Os, Cfg::OWN_STAGE ? C * Cfg::OP : 8, 4)
  COTTN_LDS_ARRAY(float, rows, 3 * C, 5)
  COTTN_LDS_ARRAY(float, rq, C, 6)
  Unparted un;
  fetch_argument_now(Q, K, V, s, log_decay, O, state_out, seg_states, state_in, lengths, H, G, seg_rows, N, units, inv_eps,
                     flags);
  constexpr int VALUE_PARTS = LDV / DV;   // (several only where sequences are few: nothing past the caches)
  const bool carried = flags & CARRIED, stream_q = VALUE_PARTS == 1 && (flags & STREAM_Q),
             stream_kv = VALUE_PARTS == 1 && (flags & STREAM_KV);
  int unit, seg, part = 0, row_begin, row_count;
  if constexpr (VALUE_PARTS > 1) {   // (one segment, whose rows are dealt to workgroups, seg_rows to the first: row_part)
    unit = blockIdx.x / VALUE_PARTS;
    part = blockIdx.x % VALUE_PARTS;
    seg = unit / units;
    unit -= seg * units;
    row_part(seg, seg_rows / C, row_begin, row_count);
    row_begin *= C;
    row_count *= C;
  } else {
    unit_and_segment(blockIdx.x, units, G, unit, seg);
    row_begin = seg * seg_rows;
    row_count = seg_rows;
  }
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int rg = w % RG, cp = w / RG;
  const elem_t* Qu = Q + size_t(unit) * N * DK;
  const elem_t* Ku = K + size_t(unit) * N * DK;
  const elem_t* Vu = V + size_t(unit) * N * LDV + part * DV;
  elem_t* Ou = O + size_t(unit) * N * LDV + part * DV;
  const int there = valid_rows(lengths, unit, H, N), piece_end = min(N, row_begin + row_count);
  const int row_end = max(row_begin, min(there, piece_end));
  const bool ends_here = there > row_begin ? there <= piece_end : there == 0 && seg == 0;   // the state after the last row
  const int scan_begin = VALUE_PARTS > 1 ? 0 : row_begin;   // rows before row_begin only make the state
  if (there <= row_begin && !ends_here) {
    zero_rows<DV, LDV>(Ou, row_begin, piece_end);
    return;
  }
  StageK qst, kst;
  StageV vst;
  if (scan_begin == row_begin) qst.fetch(Qu, row_begin, row_end, stream_q);
  kst.fetch(Ku, scan_begin, row_end, stream_kv);
  vst.fetch(Vu, scan_begin, row_end, stream_kv);
  const int head = unit - quotient(unit, H) * H.n;
  const Decay g(log_decay[head]);
  const float scale = s[lengths != nullptr ? unit : head];

  f32x4 sacc[ST::NCT][ST::NRT];
#pragma unroll
  for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
    for (int y = 0; y < ST::NRT; ++y) sacc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool active = ST::active(w);
  if (VALUE_PARTS == 1 && active && seg > 0) {
    const float* slots = seg_states + size_t(unit) * G.n * DK * DV;
    add_decayed_states<false>(sacc, carried ? seg : 0, carried ? seg : seg - 1, g, seg_rows, [&](int slot, int x, int y) {
      return *reinterpret_cast<const f32x4*>(slots + size_t(slot) * DK * DV +
                                             tiled_state_offset(ST::col_tile(w, x), ST::row_tile(w, y), DV / 16, l));
    });
  }
  bool infinite = false;
  if (active && state_in != nullptr) {
    const float since = STATE_UNIT * g.after(float(scan_begin));
    const float* src = state_in + size_t(unit) * DK * LDV + part * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(src + (16 * ST::col_tile(w, x) + r) * LDV +
                                                        16 * ST::row_tile(w, y) + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) sacc[x][y][v] = __builtin_fmaf(since, t[v], sacc[x][y][v]);
      }
    infinite = any_infinite(sacc);
  }

  const float row = float(16 * rg + r);            // of the chunk: this lane's query
  const float to_row = g.after(row + 1.f);         // from the state before the chunk
  float on_diagonal[4];                            // g^(i-j) in the tile of the wave's own rows, 0 above the diagonal
#pragma unroll
  for (int v = 0; v < 4; ++v) on_diagonal[v] = 4 * q4 + v <= r ? g.after(float(r - 4 * q4 - v)) : 0.f;
  const Kept whole_chunk(g, float(C));
  RowPieces<DV, NOT> finished;   // rows of the chunk before, stored one chunk late
#pragma unroll
  for (int j = 0; j < RowPieces<DV, NOT>::PER_LANE; ++j) finished.v[j] = uint4{0u, 0u, 0u, 0u};
  void* stage = Cfg::OWN_STAGE ? static_cast<void*>(Os + 16 * rg * Cfg::OP) : static_cast<void*>(Qs + 16 * rg * TPK);
  const int col0 = 16 * NOT * cp;
  for (int row0 = scan_begin; row0 < row_end; row0 += C) {
    const int n = min(C, row_end - row0);
    const bool mine = VALUE_PARTS == 1 || row0 >= row_begin;
    if (active) {
      if (mine) {
#pragma unroll
        for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
          for (int y = 0; y < ST::NRT; ++y)
            store4_lds(Sl + (16 * ST::col_tile(w, x) + r) * SP + 16 * ST::row_tile(w, y) + 4 * q4, PER_UNIT * sacc[x][y][0],
                       PER_UNIT * sacc[x][y][1], PER_UNIT * sacc[x][y][2], PER_UNIT * sacc[x][y][3], un);
      }
      (n == C ? whole_chunk : Kept(g, float(n))).on(sacc, infinite);
    }
    {
      RowFactors<StageK> f;
      if (mine) {
        f.commit(qst, Qs, inv_eps, un);
        qst.store_rinv(rq, f.left);
      }
      f.commit(kst, Ks, inv_eps, un);
      store_key_factors<StageK, C>(rows, f, g, n);
      vst.commit_plain(Vs, un);
    }
    if (row0 + C < row_end) {
      if (VALUE_PARTS == 1 || row0 + C >= row_begin) qst.fetch(Qu, row0 + C, row_end, stream_q);
      kst.fetch(Ku, row0 + C, row_end, stream_kv);
      vst.fetch(Vu, row0 + C, row_end, stream_kv);
    }
    if (row0 > row_begin) store_row_pieces<DV, NOT, LDV>(finished, Ou, row0 - C + 16 * rg, row_end, l, col0);
    __syncthreads();

    f32x4 oacc[NOT];
    if (mine) {
      // what the state gives: O^T = S^T Q^T, then the row's factor
      frag8 qf[Cfg::KSK];
#pragma unroll
      for (int ks = 0; ks < Cfg::KSK; ++ks) qf[ks] = lds_row_frag(Qs + (16 * rg + r) * TPK + 32 * ks, q4);
      const float ri = rq[16 * rg + r];
#pragma unroll
      for (int nt = 0; nt < NOT; ++nt) oacc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < Cfg::KSK; ++ks) {
        frag8 sf[NOT];
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt) sf[nt] = lds_col_frag_ks(Sl, SP, ks, q4, col0 + 16 * nt, r);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt) oacc[nt] = mma16(sf[nt], qf[ks], oacc[nt]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int nt = 0; nt < NOT; ++nt)
#pragma unroll
        for (int v = 0; v < 4; ++v) oacc[nt][v] *= ri * to_row;

      // the chunk itself, 32 tokens at a time
#pragma unroll
      for (int p = 0; p < Cfg::NP; ++p) {
        if (2 * p > rg) break;   // wave-uniform: every key is masked from here on
        const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
        frag8 vc[NOT], kr[2][Cfg::KSK];
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt) vc[nt] = lds_col_frag(Vs, TPV, t0, t1, col0 + 16 * nt, r);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) kr[half][ks] = lds_row_frag(Ks + (16 * (2 * p + half) + r) * TPK + 32 * ks, q4);
        __builtin_amdgcn_sched_barrier(0);
        frag8 pf;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int jt = 2 * p + half;
          f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < Cfg::KSK; ++ks) t = mma16(kr[half][ks], qf[ks], t);
          // t[v] = q_(16 rg + r) . k_(16 jt + 4 q4 + v), a row's factor at a time (decay.h: RowFactors)
          const f32x4 kj = *reinterpret_cast<const f32x4*>(rows + (jt == rg ? 0 : C) + 16 * jt + 4 * q4);
          const float below = ri * g.after(row - float(16 * jt + 15));   // (jt < rg)
#pragma unroll
          for (int v = 0; v < 4; ++v) t[v] = jt > rg ? 0.f : t[v] * kj[v] * (jt == rg ? ri * on_diagonal[v] : below);
          put_four(pf, half, t);
        }
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt) oacc[nt] = mma16_add(vc[nt], pf, oacc[nt]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // the state after the chunk, if somebody takes it
    if (active && (row0 + C < row_end || (state_out != nullptr && ends_here))) {
      const WeightedTile<ST, Cfg::NP, TPK, PARTS> k(Ks, rows + 2 * C, w, r, q4);
      constexpr int YN = ST::NRT < 4 ? ST::NRT : 4;
#pragma unroll
      for (int y0 = 0; y0 < ST::NRT; y0 += YN)
        k.template add<YN, TPV>(Vs, y0, w, r, q4, [&](int x, int y) -> f32x4& { return sacc[x][y0 + y]; });
    }
    if (mine) {
      wave_lds_sync();
      gather_rows_transposed<DV, NOT>(oacc, scale, stage, l, finished, un, col0);
    }
    __syncthreads();   // everything of the chunk is read
  }
  if (row_end > row_begin)
    store_row_pieces<DV, NOT, LDV>(finished, Ou, row_begin + (row_end - row_begin - 1) / C * C + 16 * rg, row_end, l, col0);
  if (lengths != nullptr) zero_rows<DV, LDV>(Ou, row_end, piece_end);
  if (state_out != nullptr && ends_here && active) {
    float* out = state_out + size_t(unit) * DK * LDV + part * DV;
#pragma unroll
    for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
      for (int y = 0; y < ST::NRT; ++y)
        *reinterpret_cast<f32x4*>(out + (16 * ST::col_tile(w, x) + r) * LDV + 16 * ST::row_tile(w, y) + 4 * q4) =
            PER_UNIT * sacc[x][y];
  }
}

template <int DK, int DV, int C, int CS, int LDV = DV>
hipError_t run_fwd_decay(const DecayArgs& a) {
  const int units = a.B * a.H;
  float* states = static_cast<float*>(a.workspace);
  if (a.G > 1) {
    hipError_t err = COTTN_SYM(launch_decay_totals)(a, states);
    if (err == hipSuccess && a.carried) err = launch_decay_carry(a, states, false);
    if (err != hipSuccess) return err;
  }
  // Rows that nothing finds in a cache again, as without decay (fwd_causal_bf16.hip): 64 x 16 heads of 2048 rows, forward
  // alone, 128 x 128 561 -> 558 us, 64 x 64 228.5 -> 223.4; where they fit, 96 units of 1024 rows 64 x 64 with backward 63.7 ->
  // 64.1.
  const double bytes = 2.0 * units * double(a.N) * (DK + LDV) * ELEM;
  const int flags = (a.carried ? CARRIED : 0) | (bytes > 256.0 * 1024 * 1024 ? STREAM_Q : 0) |
                    (a.G == 1 && bytes > 1024.0 * 1024 * 1024 ? STREAM_KV : 0);
  const auto scan = [&](auto kernel) {
    return launch_kernel(COTTN_SYM_STR(fwd_decay_scan), kernel, dim3(units * (LDV > DV ? LDV / DV * a.row_parts : a.G)),
                         dim3(64 * (C / 16) * CS), 0, a.stream,
                         static_cast<const elem_t*>(a.Q), static_cast<const elem_t*>(a.K), static_cast<const elem_t*>(a.V), a.s,
                         a.log_decay, static_cast<elem_t*>(a.O), a.state, states, a.state_in, a.seq_len, Divisor(a.H),
                         Divisor(a.G), LDV > DV ? a.part_rows : a.seg_rows, a.N, units, 1.0f / a.eps, flags);
  };
  if (a.state != nullptr) return scan(COTTN_SYM(fwd_decay_scan)<DK, DV, C, CS, EXACT_PARTS, LDV>);
  return scan(COTTN_SYM(fwd_decay_scan)<DK, DV, C, CS, ROUNDED_PARTS, LDV>);
}

template <int DK, int DV, int C>
hipError_t run_decay_totals(const DecayArgs& a, float* dst) {
  // 128 rows at a time where segments are that long: eight waves, a key tile each (96 units of 1024 rows forward + backward
  // 162.5 -> 156.4 us; not at narrower shapes, 64 x 64 63.6 / 63.9, 32 x 32 35.8 / 37.1, 128 x 64 105.7 / 106.7)
  if constexpr (C == 64 && !ELEM_IS_F32 && DK == 128 && DV == 128)
    if (a.seg_rows >= 128) return run_decay_totals<DK, DV, 128>(a, dst);
  const int units = a.B * a.H;
  return launch_kernel(COTTN_SYM_STR(decay_segment_state), COTTN_SYM(decay_segment_state)<DK, DV, C>, dim3(units * a.G),
                       dim3(4 * C), 0, a.stream, static_cast<const elem_t*>(a.K), static_cast<const elem_t*>(a.V), dst,
                       a.log_decay, a.seq_len, Divisor(a.H), Divisor(a.G), a.seg_rows, a.N, units, 1.0f / a.eps);
}

// In place, for four neighbouring elements: slot k (in walking order) <- what the state at its start is, which is g^seg_rows
// times that of the slot before, and that slot's total.  16 units of 32 segments 64 x 64: 7.2 us, two trips to memory a batch
// of eight slots.
__global__ __launch_bounds__(256) void decay_carry(float* __restrict__ slots, const float* __restrict__ log_decay,
                                                   const int* __restrict__ lengths, Divisor H, int G, int seg_rows, int N,
                                                   int elems, long total, int reverse) {
  const long at = (long(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= total) return;
  const int unit = int(at / elems);
  float* p = slots + size_t(unit) * G * elems + at % elems;
  const Decay g(log_decay[unit - quotient(unit, H) * H.n]);
  const Kept kept(g, float(seg_rows));
  const int there = valid_rows(lengths, unit, H, N), n = max(1, (there + seg_rows - 1) / seg_rows);   // segments with rows
  constexpr int BATCH = 8;
  f32x4 run = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < n; k0 += BATCH) {
    f32x4 t[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      t[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k0 + i + 1 < n) t[i] = *reinterpret_cast<const f32x4*>(p + size_t(reverse ? n - 1 - k0 - i : k0 + i) * elems);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (k0 + i >= n) break;
      *reinterpret_cast<f32x4*>(p + size_t(reverse ? n - 1 - k0 - i : k0 + i) * elems) = run;
      run = kept.of(run) + t[i];
    }
  }
}

}  // namespace
}  // namespace COTTN_NS

using namespace COTTN_NS;

#define COTTN_DECAY_SHAPES(CASE)                                                                                     \
  switch (a.dk * 1000 + a.dv) {                                                                                      \
    CASE(32, 32) CASE(32, 64) CASE(32, 128) CASE(64, 32) CASE(64, 64) CASE(64, 128) CASE(128, 32) CASE(128, 64)      \
    CASE(128, 128)                                                                                                   \
    default: return hipErrorInvalidValue;                                                                            \
  }

// Rows of a chunk: 64, in fp32 32.  Waves on a row group: one; two where the output of a wave would be 128 columns wide and in
// fp32, whose chunk is two row groups; in fp32 128 x 128, where the LDS holds one workgroup to a compute unit, four (two /
// four: 384 units of 512 rows 330 / 284 us, 15 of 777 43.0 / 41.4; 64 x 64, 15 units of 777, 128 registers for two workgroups
// of eight waves, 18.7 / 21.7). 16-bit 128 x 128 with more workgroups than compute units: 32 rows, so that two of them share
// one (1024 units of 2048 rows, 64 / 32 rows 598 / 555 us; 192 workgroups of 512 rows each, with totals and backward, 157 /
// 163; 32 rows with four waves, spilling, 1187).
hipError_t COTTN_SYM(fwd_decay)(const DecayArgs& a) {
  constexpr int C = ELEM_IS_F32 ? 32 : 64, CS = ELEM_IS_F32 ? 2 : 1;
  switch (a.value_columns != a.dv ? (a.dk * 1000 + a.dv) * 100 + a.value_columns : 0) {
    case 3206432: return run_fwd_decay<32, 32, C, CS, 64>(a);
    case 6406432: return run_fwd_decay<64, 32, C, CS, 64>(a);
    case 12806432: return run_fwd_decay<128, 32, C, CS, 64>(a);
    case 3212832: return run_fwd_decay<32, 32, C, CS, 128>(a);
    case 6412832: return run_fwd_decay<64, 32, C, CS, 128>(a);
    case 12812832: return run_fwd_decay<128, 32, C, CS, 128>(a);
    case 3212864: return run_fwd_decay<32, 64, C, CS, 128>(a);
    case 6412864: return run_fwd_decay<64, 64, C, CS, 128>(a);
    case 12812864: return run_fwd_decay<128, 64, C, CS, 128>(a);
    default: break;
  }
#ifndef COTTN_ELEM_F32
  if (a.dk == 128 && a.dv == 128 && long(a.B) * a.H * a.G > 256) return run_fwd_decay<128, 128, 32, 2>(a);
#endif
#define COTTN_CASE(DK, DV) \
  case DK * 1000 + DV: return run_fwd_decay<DK, DV, ELEM_IS_F32 ? 32 : 64, DK == 128 && DV == 128 ? (ELEM_IS_F32 ? 4 : 2) : ELEM_IS_F32 ? 2 : 1>(a);
  COTTN_DECAY_SHAPES(COTTN_CASE)
#undef COTTN_CASE
}

hipError_t COTTN_SYM(launch_decay_totals)(const DecayArgs& a, float* dst) {
#define COTTN_CASE(DK, DV) \
  case DK * 1000 + DV: return run_decay_totals<DK, DV, 64>(a, dst);
  COTTN_DECAY_SHAPES(COTTN_CASE)
#undef COTTN_CASE
}

#if !defined(COTTN_ELEM_F16) && !defined(COTTN_ELEM_F32)   // not specific to the element type
hipError_t launch_decay_carry(const DecayArgs& a, float* slots, bool reverse) {
  const int elems = a.dk * a.dv;
  const long total = long(a.B) * a.H * elems;
  return launch_kernel("decay_carry", decay_carry, dim3(unsigned((total / 4 + 255) / 256)), dim3(256), 0, a.stream, slots,
                       a.log_decay, a.seq_len, Divisor(a.H), a.G, a.seg_rows, a.N, elems, total, int(reverse));
}
#endif

}  // namespace cottn
