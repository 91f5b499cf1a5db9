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

// A workgroup of four waves takes COLS value columns of a (batch, head).  RG row groups of 16 tokens, 4 / RG waves on each,
// which share its output columns.
template <int DK, int DV, int COLS, int RG>
__global__ __launch_bounds__(256) void COTTN_SYM(tree_kernel)(
    const elem_t* __restrict__ q, const elem_t* __restrict__ k, const elem_t* __restrict__ v, const float* __restrict__ s,
    const float* __restrict__ log_decay, const int* __restrict__ parent, const float* __restrict__ state,
    elem_t* __restrict__ o, Divisor H, int n_tokens, float inv_eps, int stream) {
  constexpr int T = 16 * RG < 32 ? 32 : 16 * RG;   // rows of the tiles: a product takes 32 tokens
  constexpr int CS = 4 / RG, COL_TILES = COLS / 16, NOT = COL_TILES / CS < 1 ? 1 : COL_TILES / CS;
  constexpr int TPK = tile_pitch(DK, T), TPV = tile_pitch(COLS, T), SP = lds_pitch(COLS), KSK = DK / 32, PARTS = DV / COLS;
  using StageK = TileStage<DK, T, 256>;
  using StageV = TileStage<COLS, T, 256, DV>;
  constexpr int STAGE = stage_pitch(COLS);
  __shared__ __attribute__((aligned(16))) lds_t Qs[T * TPK], Ks[T * TPK], Vs[T * TPV], Sl[DK * SP];
  __shared__ __attribute__((aligned(16))) elem_t Os[RG * 16 * STAGE];
  __shared__ __attribute__((aligned(16))) float rq[T], rk[T], depth[64];
  __shared__ unsigned long long paths[64];
  Unparted un;
  fetch_argument_now(q, k, v, s, log_decay, parent, state, o, H, n_tokens, inv_eps, stream);
  const int unit = blockIdx.x / PARTS, part = blockIdx.x % PARTS, b = quotient(unit, H), head = unit - b * H.n;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int rg = w % RG, cp = w / RG;

  // the state, four columns of a row to a thread
  constexpr int TPR = COLS / 4, RPP = 256 / TPR, PASSES = (DK + RPP - 1) / RPP;
  const float* S = state + size_t(unit) * DK * DV + part * COLS;
  f32x4 srows[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int row = p * RPP + tid / TPR;
    srows[p] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (DK % RPP == 0 || row < DK) {
      const f32x4* at = reinterpret_cast<const f32x4*>(S + size_t(row) * DV + tid % TPR * 4);
      srows[p] = stream ? __builtin_nontemporal_load(at) : *at;
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
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int row = p * RPP + tid / TPR;
    if (DK % RPP == 0 || row < DK) store4_lds(Sl + row * SP + tid % TPR * 4, srows[p][0], srows[p][1], srows[p][2], srows[p][3], un);
  }
  __syncthreads();
  if (cp * NOT >= COL_TILES || 16 * rg >= n_tokens) return;

  const int col0 = 16 * NOT * cp;
  frag8 qf[KSK];
#pragma unroll
  for (int ks = 0; ks < KSK; ++ks) qf[ks] = lds_row_frag(Qs + (16 * rg + r) * TPK + 32 * ks, q4);
  f32x4 oacc[NOT];
#pragma unroll
  for (int nt = 0; nt < NOT; ++nt) oacc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < KSK; ++ks)
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt) oacc[nt] = mma16(lds_col_frag_ks(Sl, SP, ks, q4, col0 + 16 * nt, r), qf[ks], oacc[nt]);
  const unsigned long long path = paths[16 * rg + r];
  const float mine = depth[16 * rg + r], ri = rq[16 * rg + r], since = ri * g.after(mine + 1.f);
#pragma unroll
  for (int nt = 0; nt < NOT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) oacc[nt][i] *= since;
#pragma unroll
  for (int p = 0; p < T / 32; ++p) {
    if (2 * p > rg) break;   // parents come before their children
    const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
    frag8 pf;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int j = 32 * p + 16 * half + 4 * q4;   // this lane's keys j .. j + 3
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KSK; ++ks) t = mma16(lds_row_frag(Ks + (32 * p + 16 * half + r) * TPK + 32 * ks, q4), qf[ks], t);
      const f32x4 rj = *reinterpret_cast<const f32x4*>(rk + j), dj = *reinterpret_cast<const f32x4*>(depth + j);
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = (path >> (j + i)) & 1 ? t[i] * (ri * rj[i] * g.after(mine - dj[i])) : 0.f;
      put_four(pf, half, t);
    }
#pragma unroll
    for (int nt = 0; nt < NOT; ++nt) oacc[nt] = mma16_add(lds_col_frag(Vs, TPV, t0, t1, col0 + 16 * nt, r), pf, oacc[nt]);
  }
  RowPieces<COLS, NOT> done;
  gather_rows_transposed<COLS, NOT>(oacc, scale, Os + 16 * rg * STAGE, l, done, un, col0);
  store_row_pieces<COLS, NOT, DV>(done, o + size_t(unit) * n_tokens * DV + part * COLS, 16 * rg, n_tokens, l, col0);
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
