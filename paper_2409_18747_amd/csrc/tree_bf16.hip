// A tree of up to 64 drafted tokens over the state of its sequence (gfx950): with g = exp(log_decay[h]) and depths counted from
// the roots,
//     o_i = s [ g^(depth_i + 1) qh_i S + sum over j = i and its ancestors of g^(depth_i - depth_j) (qh_i . kh_j) v_j ].
// The state is read once and stays.  This file builds the bfloat16 kernel, the IEEE half one when it is included with
// COTTN_ELEM_F16 defined and the fp32 one with COTTN_ELEM_F32 and COTTN_F32_WHOLE.
#include "device_common.h"
#include "launch.h"
#include "tile_io.h"
#include "decay.h"

namespace cottn {
namespace COTTN_NS {
namespace {

// Operand fragment down the columns of a row-major tile like lds_col_frag, where the 16 columns are four groups of four, STRIDE
// apart: column m of the fragment is column col0 + STRIDE (m / 4) + m % 4 of the tile.
template <int STRIDE>
__device__ __forceinline__ frag8 lds_spread_frag(const lds_t* tile, int pitch, int k0, int k1, int col0, int r) {
#ifdef COTTN_F32_WHOLE
  return lds_col_frag(tile, pitch, k0, k1, col0 + STRIDE * (r / 4) + r % 4 - r, r);
#else
  const lds_t* at = tile + col0 + STRIDE * (r & 3);
  const s16x4 lo = lds_read_tr(at + (k0 + (r >> 2)) * pitch), hi = lds_read_tr(at + (k1 + (r >> 2)) * pitch);
  return __builtin_bit_cast(frag8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
#endif
}

// A workgroup of four waves takes COLS value columns of a (batch, head): RG row groups of 16 tokens, of which a wave has a part
// of the columns (NOT tiles) of every one, or of every RW-th where there are fewer than four column tiles.  Each masked tile is
// formed by one wave and handed on as the fragment that it enters the next product as.  The columns of a wave's two tiles are
// interleaved by fours, so that a lane ends with eight consecutive columns of a row, a whole 16-byte store.
//   The state is most of what is read, and what bounds a call of many sequences.  It is requested first.  Up to 32 tokens its
// rows go through the LDS; beyond, where the tiles of the rows would then leave a compute unit one workgroup, every wave reads
// its columns straight into operand fragments (DIRECT), 64-byte pieces of rows.  1024 states of 128 x 128, through the LDS /
// direct, when that was chosen: 13 tokens 15.1 / 17.1 us, 64 tokens 30.3 / 28.5 (one workgroup to a compute unit 35.5).  As it
// is, 64 tokens 27.0 us for 134 MB, 5.0 TB/s; fp32, whose 128 columns are two workgroups that each read the rows and form the
// masked tiles, 13 tokens 28.6 us for 94 MB, 64 tokens 95.7 for 201 MB.
template <int DK, int DV, int COLS, int RG>
struct TreeCfg {
  static constexpr int T = 16 * RG < 32 ? 32 : 16 * RG, PAIRS = T / 32;   // rows of the tiles: a product takes 32 tokens
  static constexpr int COL_TILES = COLS / 16, NOT = COL_TILES < 4 ? 1 : COL_TILES / 4, CW = COL_TILES / NOT, RW = 4 / CW;
  static constexpr int RGW = RG / RW < 1 ? 1 : RG / RW;   // row groups of a wave
  static constexpr int TPK = tile_pitch(DK, T), TPV = tile_pitch(COLS, T), SP = lds_pitch(COLS), KSK = DK / 32;
  static constexpr bool DIRECT = RG > 2;
  // columns of a wave's tile nt: col0 + STRIDE (m / 4) + OFFSET nt + m % 4
  static constexpr int STRIDE = DIRECT ? 4 : 4 * NOT, OFFSET = DIRECT ? 16 : 4;
  static constexpr int LDS_BYTES = LDS_ELEM * (2 * T * TPK + T * TPV + (DIRECT ? 8 : DK * SP)) + int(sizeof(frag8)) * RG * PAIRS * 64 + 2048;
  static constexpr int AT_ONCE = LDS_BYTES <= 80 * 1024 ? 2 : 1;
};
template <int DK, int DV, int COLS, int RG>
__global__ __launch_bounds__(256, (TreeCfg<DK, DV, COLS, RG>::AT_ONCE)) void COTTN_SYM(tree_kernel)(
    const elem_t* __restrict__ q, const elem_t* __restrict__ k, const elem_t* __restrict__ v, const float* __restrict__ s,
    const float* __restrict__ log_decay, const int* __restrict__ parent, const float* __restrict__ state,
    elem_t* __restrict__ o, Divisor H, int n_tokens, float inv_eps, int stream) {
  using Cfg = TreeCfg<DK, DV, COLS, RG>;
  constexpr int T = Cfg::T, PAIRS = Cfg::PAIRS, NOT = Cfg::NOT, CW = Cfg::CW, RW = Cfg::RW, RGW = Cfg::RGW, KSK = Cfg::KSK;
  constexpr int TPK = Cfg::TPK, TPV = Cfg::TPV, SP = Cfg::SP, PARTS = DV / COLS, STRIDE = Cfg::STRIDE, OFFSET = Cfg::OFFSET;
  constexpr bool DIRECT = Cfg::DIRECT;
  static_assert(NOT <= 2, "a lane stores eight columns at most");
  using StageK = TileStage<DK, T, 256>;
  using StageV = TileStage<COLS, T, 256, DV>;
  __shared__ __attribute__((aligned(16))) lds_t Ks[T * TPK], Vs[T * TPV], Sl[DIRECT ? 8 : DK * SP];
  // the query rows; direct: finished rows are staged here when those are read
  constexpr int OP = stage_pitch(COLS), Q_ROOM = LDS_ELEM * T * TPK, O_ROOM = DIRECT ? ELEM * 16 * RG * OP : 0;
  __shared__ __attribute__((aligned(16))) char room[Q_ROOM > O_ROOM ? Q_ROOM : O_ROOM];
  lds_t* Qs = reinterpret_cast<lds_t*>(room);
  __shared__ __attribute__((aligned(16))) frag8 Ps[RG][PAIRS][64];   // masked tiles: row group, 32 keys, lane
  __shared__ __attribute__((aligned(16))) float rq[T], rk[T], depth[64];
  __shared__ unsigned long long paths[64];
  Unparted un;
  fetch_argument_now(q, k, v, s, log_decay, parent, state, o, H, n_tokens, inv_eps, stream);
  const int unit = blockIdx.x / PARTS, part = blockIdx.x % PARTS, b = quotient(unit, H), head = unit - b * H.n;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;

  const int cw = w % CW, rw = RW == 1 ? 0 : w / CW, col0 = 16 * NOT * cw;   // this wave's columns, of row groups rw, rw + RW, ..
  const float* S = state + size_t(unit) * DK * DV + part * COLS;
  const auto read = [&](const auto* at) { return stream ? __builtin_nontemporal_load(at) : *at; };
  // through the LDS: four columns of a row to a thread
  constexpr int TPR = COLS / 4, RPP = 256 / TPR, PASSES = (DK + RPP - 1) / RPP;
  f32x4 srows[DIRECT ? 1 : PASSES];
  // direct: key slots of 32 ks .., columns col0 + 16 nt + r
  float sv[DIRECT ? NOT : 1][DIRECT ? KSK : 1][8];
  if constexpr (DIRECT) {
#pragma unroll
    for (int ks = 0; ks < KSK; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt)
          sv[nt][ks][j] = read(S + (32 * ks + (j < 4 ? slot_lo(q4) + j : slot_hi(q4) + j - 4)) * DV + col0 + 16 * nt + r);
  } else {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int row = p * RPP + tid / TPR;
      srows[p] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (DK % RPP == 0 || row < DK) srows[p] = read(reinterpret_cast<const f32x4*>(S + row * DV + tid % TPR * 4));
    }
  }
  StageK qst, kst;
  StageV vst;
  qst.fetch(q + size_t(unit) * n_tokens * DK, 0, n_tokens);
  kst.fetch(k + size_t(unit) * n_tokens * DK, 0, n_tokens);
  vst.fetch(v + size_t(unit) * n_tokens * DV + part * COLS, 0, n_tokens);
  const Decay g(log_decay != nullptr ? log_decay[head] : 0.f);
  const float scale = s[head];
  if (w == 0) {
    const TreeNode node(parent + size_t(b) * n_tokens, n_tokens, l);
    paths[l] = node.path;
    depth[l] = float(node.depth());
  }
  {
    RowFactors<StageK> f;
    f.commit(qst, Qs, inv_eps, un);
    qst.store_rinv(rq, f.left);
    f.commit(kst, Ks, inv_eps, un);
    kst.store_rinv(rk, f.left);
    vst.commit_plain(Vs, un);
  }
  if constexpr (!DIRECT) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int row = p * RPP + tid / TPR;
      if (DK % RPP == 0 || row < DK) store4_lds(Sl + row * SP + tid % TPR * 4, srows[p][0], srows[p][1], srows[p][2], srows[p][3], un);
    }
  }
  __syncthreads();

  // masked tiles, the pairs (row group, 32 keys) dealt to the waves; parents come before their children
#pragma unroll
  for (int rg = 0; rg < RG; ++rg)
#pragma unroll
    for (int p = 0; p < PAIRS; ++p) {
      if (2 * p > rg || (rg + p) % 4 != w || 16 * rg >= n_tokens) continue;
      const unsigned long long path = paths[16 * rg + r];
      const float mine = depth[16 * rg + r], ri = rq[16 * rg + r];
      frag8 pf, qf[KSK], kf[2][KSK];
#pragma unroll
      for (int ks = 0; ks < KSK; ++ks) qf[ks] = lds_row_frag(Qs + (16 * rg + r) * TPK + 32 * ks, q4);
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int ks = 0; ks < KSK; ++ks)
          if (2 * p + half <= rg) kf[half][ks] = lds_row_frag(Ks + (32 * p + 16 * half + r) * TPK + 32 * ks, q4);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
        if (2 * p + half <= rg) {
          const int j = 32 * p + 16 * half + 4 * q4;   // this lane's keys j .. j + 3
#pragma unroll
          for (int ks = 0; ks < KSK; ++ks) t = mma16(kf[half][ks], qf[ks], t);
          // (a row's factor at a time: decay.h, RowFactors)
          const f32x4 rj = *reinterpret_cast<const f32x4*>(rk + j), dj = *reinterpret_cast<const f32x4*>(depth + j);
#pragma unroll
          for (int i = 0; i < 4; ++i) t[i] = (path >> (j + i)) & 1 ? t[i] * rj[i] * (ri * g.after(mine - dj[i])) : 0.f;
        }
        put_four(pf, half, t);
      }
      Ps[rg][p][l] = pf;
    }
  // what the state gives, O^T = S^T Q^T, and the rows' factors
  f32x4 oacc[RGW][NOT];
#pragma unroll
  for (int i = 0; i < RGW; ++i)
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt) oacc[i][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < KSK; ++ks) {
    frag8 sf[NOT], qf[RGW];
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt) {
      if constexpr (DIRECT) {
        put_four(sf[nt], 0, f32x4{sv[nt][ks][0], sv[nt][ks][1], sv[nt][ks][2], sv[nt][ks][3]});
        put_four(sf[nt], 1, f32x4{sv[nt][ks][4], sv[nt][ks][5], sv[nt][ks][6], sv[nt][ks][7]});
      } else {
        sf[nt] = lds_spread_frag<STRIDE>(Sl, SP, 32 * ks + slot_lo(q4), 32 * ks + slot_hi(q4), col0 + OFFSET * nt, r);
      }
    }
#pragma unroll
    for (int i = 0; i < RGW; ++i)
      if (rw + i * RW < RG) qf[i] = lds_row_frag(Qs + (16 * (rw + i * RW) + r) * TPK + 32 * ks, q4);
#pragma unroll
    for (int i = 0; i < RGW; ++i)
      if (rw + i * RW < RG) {
#pragma unroll
        for (int nt = 0; nt < NOT; ++nt) oacc[i][nt] = mma16(sf[nt], qf[i], oacc[i][nt]);
      }
  }
#pragma unroll
  for (int i = 0; i < RGW; ++i) {
    if (rw + i * RW >= RG) break;
    const int row = 16 * (rw + i * RW) + r;
    const float since = rq[row] * g.after(depth[row] + 1.f);
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) oacc[i][nt][e] *= since;
  }
  __syncthreads();   // the masked tiles are there, and the query rows are read
#pragma unroll
  for (int p = 0; p < PAIRS; ++p) {
    frag8 vc[NOT];
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt) vc[nt] = lds_spread_frag<STRIDE>(Vs, TPV, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, col0 + OFFSET * nt, r);
#pragma unroll
    for (int i = 0; i < RGW; ++i) {
      const int rg = rw + i * RW;
      if (2 * p > rg || rg >= RG || 16 * rg >= n_tokens) continue;
      const frag8 pf = Ps[rg][p][l];
#pragma unroll
      for (int nt = 0; nt < NOT; ++nt) oacc[i][nt] = mma16_add(vc[nt], pf, oacc[i][nt]);
    }
  }
  // oacc[i][nt][e] = O[token 16 rg + r][value col0 + STRIDE q4 + OFFSET nt + e]
  elem_t* out = o + size_t(unit) * n_tokens * DV + part * COLS;
#pragma unroll
  for (int i = 0; i < RGW; ++i) {
    const int rg = rw + i * RW, row = 16 * rg + r;
    if (rg >= RG || 16 * rg >= n_tokens) break;
    if constexpr (DIRECT) {
      RowPieces<COLS, NOT> done;
      gather_rows_transposed<COLS, NOT>(oacc[i], scale, reinterpret_cast<elem_t*>(room) + 16 * rg * OP, l, done, un, col0);
      store_row_pieces<COLS, NOT, DV>(done, out, 16 * rg, n_tokens, l, col0);
    } else if (row < n_tokens) {
      elem_t* to = out + row * DV + col0 + STRIDE * q4;
#ifndef COTTN_ELEM_F32
      if constexpr (NOT == 2) {
        store_streaming(to, uint4{pack2(scale * oacc[i][0][0], scale * oacc[i][0][1]), pack2(scale * oacc[i][0][2], scale * oacc[i][0][3]),
                                  pack2(scale * oacc[i][1][0], scale * oacc[i][1][1]), pack2(scale * oacc[i][1][2], scale * oacc[i][1][3])});
        continue;
      }
#endif
#pragma unroll
      for (int nt = 0; nt < NOT; ++nt)
        store4(to + OFFSET * nt, scale * oacc[i][nt][0], scale * oacc[i][nt][1], scale * oacc[i][nt][2], scale * oacc[i][nt][3]);
    }
  }
}

template <int DK, int DV, int COLS, int RG>
hipError_t launch_tree(const TreeArgs& a) {
  const int units = a.B * a.H;
  const int stream = double(units) * DK * DV * sizeof(float) > 32.0 * 1024 * 1024 ? 1 : 0;
  return launch_kernel(COTTN_SYM_STR(tree_kernel), COTTN_SYM(tree_kernel)<DK, DV, COLS, RG>, dim3(units * (DV / COLS)), dim3(256), 0,
                       a.stream, static_cast<const elem_t*>(a.q), static_cast<const elem_t*>(a.k), static_cast<const elem_t*>(a.v),
                       a.s, a.log_decay, a.parent, a.state, static_cast<elem_t*>(a.o), Divisor(a.H), a.n_tokens, 1.0f / a.eps,
                       stream);
}
template <int DK, int DV>
hipError_t run_tree(const TreeArgs& a) {
  constexpr int COLS = ELEM_IS_F32 && DV == 128 ? 64 : DV;   // (four fp32 tiles of 128 columns do not fit the LDS)
  // Up to 64 states: parts of the value columns to a workgroup, so that more compute units have one.  Kernel alone, states of
  // 128 x 128, whole / 64 / 32 columns: 16 states, 13 tokens 4.1 / - / 3.5 us, 64 tokens 5.8 / 5.1 / 5.4; 64 states, 64 tokens
  // 6.5 / 5.3 / 7.3; 128 states, 13 tokens 4.7 / - / 5.4.
  if (DV > 32 && a.B * a.H <= 64) {
    if (a.n_tokens <= 16) return launch_tree<DK, DV, 32, 1>(a);
    if (a.n_tokens <= 32) return launch_tree<DK, DV, 32, 2>(a);
    return launch_tree<DK, DV, DV < 64 ? DV : 64, 4>(a);
  }
  if (a.n_tokens <= 16) return launch_tree<DK, DV, COLS, 1>(a);
  if (a.n_tokens <= 32) return launch_tree<DK, DV, COLS, 2>(a);
  return launch_tree<DK, DV, COLS, 4>(a);
}

}  // namespace
}  // namespace COTTN_NS

using namespace COTTN_NS;

hipError_t COTTN_SYM(tree)(const TreeArgs& a) {
#define COTTN_CASE(DK, DV) \
  case DK * 1000 + DV: return run_tree<DK, DV>(a);
  switch (a.dk * 1000 + a.dv) {
    COTTN_CASE(32, 32) COTTN_CASE(32, 64) COTTN_CASE(32, 128) COTTN_CASE(64, 32) COTTN_CASE(64, 64) COTTN_CASE(64, 128)
    COTTN_CASE(128, 32) COTTN_CASE(128, 64) COTTN_CASE(128, 128)
    default: return hipErrorInvalidValue;
  }
#undef COTTN_CASE
}

}  // namespace cottn
