// The gated delta rule, backward (formulas, precision: delta.h): a scan from the last chunk to the first that leaves Z and the
// gradient D with respect to the state behind every chunk; then, of all chunks at once, the gradients; then the sums for ds.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

// ---------------------------------------------------------------------------------------
// As the forward scan, a workgroup takes VC of the value columns: F = P^T dO' + (G_n/G) Kh D, Z = F - W^T (b F), and D in front
// of the chunk, one after the other.
template <typename T, int DK, int VC>
struct DeltaRevCfg {
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3;
  using KTile = PartTile<CHUNK, DK, IN>;
  using GTile = PartTile<CHUNK, VC, IN>;      // rows of dO
  using State = PartTile<DK, VC, LEVEL>;      // [key][value]
  using Errors = PartTile<CHUNK, VC, LEVEL>;  // [token][value]
  // the gradient behind the chunk, and when it is read X
  static constexpr int ROOM = State::SIZE > Errors::SIZE ? State::SIZE : Errors::SIZE;
  static constexpr int LDS_BYTES = 2 * (2 * KTile::SIZE + GTile::SIZE + ROOM + Errors::SIZE) + int(sizeof(ChunkRecord)) + 8 * CHUNK;
  static constexpr int GROUPS = (160 * 1024) / LDS_BYTES >= 3 ? 3 : (160 * 1024) / LDS_BYTES >= 2 ? 2 : 1;
};

template <typename T, int DK, int VC>
__global__ __launch_bounds__(256, (DeltaRevCfg<T, DK, VC>::GROUPS)) void delta_rev_scan(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ dO, const float* __restrict__ s,
    const int* __restrict__ lengths, const float* dstate, float* dstate_in, const ChunkRecord* __restrict__ records,
    const uint16_t* __restrict__ w_cols, float* __restrict__ zs, float* __restrict__ dstates, Divisor H, Divisor parts, int N,
    int units, int DV, float inv_eps) {
  using Cfg = DeltaRevCfg<T, DK, VC>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  using State = typename Cfg::State;
  using Errors = typename Cfg::Errors;
  using ST = StateTiles<DK, VC>;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, KS = DK / 32, NT = VC / 16;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Qs[KTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t Os[GTile::SIZE];
  __shared__ __attribute__((aligned(16))) uint16_t room[Cfg::ROOM];
  __shared__ __attribute__((aligned(16))) uint16_t Fs[Errors::SIZE];   // b F
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK], rq_since[CHUNK];
  uint16_t* const Ds = room;
  uint16_t* const Xs = room;   // - G X / |k|
  fetch_argument_now(Q, K, dO, s, lengths, dstate, dstate_in, records, w_cols, zs, dstates, H, parts, N, units, DV, inv_eps);
  int unit, part;
  unit_and_segment(blockIdx.x, units, parts, unit, part);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  const int there = valid_rows(lengths, unit, H, N), chunks = delta_chunks(N), steps = delta_chunks(there), col0 = part * VC;
  const T* Qu = Q + size_t(unit) * N * DK;
  const T* Ku = K + size_t(unit) * N * DK;
  const T* dOu = dO + size_t(unit) * N * DV + col0;
  const float scale = s[lengths != nullptr ? unit : unit - quotient(unit, H) * H.n];
  const int own = 16 * w + r;   // this lane's token of the chunk
  const bool active = ST::active(w);

  const auto state_at = [&](int x, int y) {
    return unsigned((16 * ST::key_tile(w, y) + r) * DV + col0 + 16 * ST::value_tile(w, x) + 4 * q4);
  };
  f32x4 D[ST::NV][ST::NK];
#pragma unroll
  for (int x = 0; x < ST::NV; ++x)
#pragma unroll
    for (int y = 0; y < ST::NK; ++y) {
      D[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (dstate != nullptr && active) D[x][y] = *reinterpret_cast<const f32x4*>(dstate + size_t(unit) * DK * DV + state_at(x, y));
    }

  RowTile<T, DK> kt, qt;
  RowTile<T, VC> gt;
  u32x4 rec_next = {0u, 0u, 0u, 0u};
  bf16x8 wf[2][LEVEL];
  const auto fetch_rows = [&](int c) {
    const int row0 = c * CHUNK;
    kt.fetch(Ku + size_t(row0) * DK, there - row0);
    qt.fetch(Qu + size_t(row0) * DK, there - row0);
    gt.fetch(dOu + size_t(row0) * DV, there - row0, DV);
    if (tid < RECORD_PIECES) rec_next = reinterpret_cast<const u32x4*>(records + size_t(unit) * chunks + c)[tid];
  };
  const auto fetch_W = [&](int c) {
    const uint16_t* from = w_cols + (size_t(unit) * chunks + c) * W_ELEMS;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < LEVEL; ++i)
        if (w_col_there(w, ks))
          wf[ks][i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(from + w_col_frag(w, ks) * 3 * 512 + i * 512 + l * 8));
  };
  if (steps > 0) {
    fetch_rows(steps - 1);
    fetch_W(steps - 1);
  }
  for (int c = steps - 1; c >= 0; --c) {
    if (active) {
      float* to = dstates + (size_t(unit) * chunks + c) * DK * DV;
#pragma unroll
      for (int x = 0; x < ST::NV; ++x)
#pragma unroll
        for (int y = 0; y < ST::NK; ++y) {
          State::store4(Ds, 16 * ST::key_tile(w, y) + r, 16 * ST::value_tile(w, x) + 4 * q4, D[x][y]);
          *reinterpret_cast<f32x4*>(to + state_at(x, y)) = D[x][y];
        }
    }
    kt.commit(Ks);
    qt.commit(Qs);
    qt.store_factors(rq, inv_eps);
    gt.commit(Os);
    if (tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[tid] = rec_next;
    __syncthreads();

    // F: what D gives, and the chunk's own rows
    f32x4 f[NT];
    if (tid < CHUNK) rq_since[tid] = scale * rec.since[tid] * rq[tid];
    {
      bf16x8 kf[KS][IN];
#pragma unroll
      for (int t = 0; t < NT; ++t) f[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        KTile::row_frag(Ks, own, 32 * ks + 8 * q4, kf[ks]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf16x8 df[LEVEL];
          State::col_frag(Ds, 32 * ks + 8 * q4, 32 * ks + 8 * q4 + 4, 16 * t, r, df);
          f[t] = mm<LEVEL>(df, kf[ks], f[t]);
        }
      }
      const float to_end = rec.rk_to_end[own], to_tile = scale * rec.rk_to_tile[own];
#pragma unroll
      for (int t = 0; t < NT; ++t) f[t] *= to_end;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (2 * p + 1 < w) continue;   // queries before the wave's keys
        f32x4 half[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int it = 2 * p + h;
          if (it >= w) {
            f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              bf16x8 qf[IN];
              KTile::row_frag(Qs, 16 * it + r, 32 * ks + 8 * q4, qf);
              t = mm<LEVEL>(qf, kf[ks], t);
            }
            const f32x4 rq4 = *reinterpret_cast<const f32x4*>(rq + 16 * it + 4 * q4);
            if (it > w) {
              half[h] = t * rq4 * (*reinterpret_cast<const f32x4*>(rec.in_tile + 16 * it + 4 * q4) * (to_tile * rec.between[it][w]));
            } else {
              const double g_own = rec.decay[own];
              const float rk_own = scale * rec.rk[own];
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const int i = 16 * it + 4 * q4 + v;
                half[h][v] = i >= own ? t[v] * rq4[v] * (rk_own * decay_between(rec.decay[i], g_own)) : 0.f;
              }
            }
          }
        }
        bf16x8 pf[LEVEL];
        split8<LEVEL>(half[0], half[1], pf);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf16x8 gf[IN];
          GTile::col_frag(Os, 32 * p + 4 * q4, 32 * p + 16 + 4 * q4, 16 * t, r, gf);
          f[t] = mm<LEVEL>(gf, pf, f[t]);
        }
      }
    }
    const float b = rec.beta[own], x_since = -b * rec.rk_since[own], times = rec.times, plus = rec.plus;
#pragma unroll
    for (int t = 0; t < NT; ++t) Errors::store4(Fs, own, 16 * t + 4 * q4, b * f[t]);
    if (c > 0) fetch_rows(c - 1);
    __syncthreads();

    {
      f32x4 z[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) z[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        if (w_col_there(w, ks)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8 ff[LEVEL];
            Errors::col_frag(Fs, 32 * ks + 8 * q4, 32 * ks + 8 * q4 + 4, 16 * t, r, ff);
            z[t] = mm<LEVEL>(ff, wf[ks], z[t]);
          }
        }
      float* to = zs + ((size_t(unit) * chunks + c) * CHUNK + own) * DV + col0 + 4 * q4;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        z[t] = f[t] - z[t];
        Errors::store4(Xs, own, 16 * t + 4 * q4, x_since * z[t]);
        *reinterpret_cast<f32x4*>(to + 16 * t) = z[t];
      }
      if (c > 0) fetch_W(c - 1);
    }
    __syncthreads();

    if (active) {
#pragma unroll
      for (int x = 0; x < ST::NV; ++x)
#pragma unroll
        for (int y = 0; y < ST::NK; ++y)
#pragma unroll
          for (int v = 0; v < 4; ++v) D[x][y][v] = __builtin_fmaf(D[x][y][v], plus, D[x][y][v] * times);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int t0 = 32 * ks + 8 * q4;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(rq_since + t0), hi = *reinterpret_cast<const f32x4*>(rq_since + t0 + 4);
        bf16x8 gf[ST::NV][LEVEL], xf[ST::NV][LEVEL];
#pragma unroll
        for (int x = 0; x < ST::NV; ++x) {
          bf16x8 raw[IN];
          GTile::col_frag(Os, t0, t0 + 4, 16 * ST::value_tile(w, x), r, raw);
          f32x4 a, b_;
          join8<IN>(raw, a, b_);
          split8<LEVEL>(a * lo, b_ * hi, gf[x]);
          Errors::col_frag(Xs, t0, t0 + 4, 16 * ST::value_tile(w, x), r, xf[x]);
        }
#pragma unroll
        for (int y = 0; y < ST::NK; ++y) {
          bf16x8 kf[IN], qf[IN];
          KTile::col_frag(Ks, t0, t0 + 4, 16 * ST::key_tile(w, y), r, kf);
          KTile::col_frag(Qs, t0, t0 + 4, 16 * ST::key_tile(w, y), r, qf);
#pragma unroll
          for (int x = 0; x < ST::NV; ++x) {
            D[x][y] = mm<LEVEL>(xf[x], kf, D[x][y]);
            D[x][y] = mm<LEVEL>(gf[x], qf, D[x][y]);
          }
        }
      }
    }
    __syncthreads();
  }
  if (dstate_in != nullptr && active) {
#pragma unroll
    for (int x = 0; x < ST::NV; ++x)
#pragma unroll
      for (int y = 0; y < ST::NK; ++y) *reinterpret_cast<f32x4*>(dstate_in + size_t(unit) * DK * DV + state_at(x, y)) = D[x][y];
  }
}

// ---------------------------------------------------------------------------------------
// The gradients of a chunk, a workgroup each.  A wave owns key columns of dQ and dK, so that it meets, and takes apart, its rows
// of H and D once; accumulators hold them transposed, four consecutive columns of a token in a lane.
template <typename T, int DK, int DV>
struct DeltaGradCfg {
  static constexpr int IN = Rows<T>::PARTS, LEVEL = 3, PAD = sizeof(T) == 4 ? 8 : 16;
  using KTile = PartTile<CHUNK, DK, IN, PAD>;
  using GTile = PartTile<CHUNK, DV, IN, PAD>;
  using ETile = PartTile<CHUNK, DV, LEVEL, PAD>;
  using MTile = PartTile<CHUNK, CHUNK, LEVEL, PAD>;
  // first the rows of dO, E and Z, then two masked tiles and the rows of K and Q
  static constexpr int FIRST = GTile::SIZE + 2 * ETile::SIZE, SECOND = 2 * MTile::SIZE + 2 * KTile::SIZE;
  static constexpr int SIZE = FIRST > SECOND ? FIRST : SECOND;
  static constexpr int LDS_BYTES = 2 * SIZE + CHUNK * 8 + 16 + int(sizeof(ChunkRecord));
  static constexpr int GROUPS = (160 * 1024) / LDS_BYTES >= 2 ? 2 : 1;
  // key tiles of a wave and token tiles that it forms of them
  static constexpr int KT = DK / 16, NK = KT >= 4 ? KT / 4 : 1, NTOK = KT >= 4 ? 4 : 2;
};

// four consecutive elements
template <typename T>
__device__ __forceinline__ f32x4 load_row4(const T* p) {
  typedef __attribute__((ext_vector_type(4))) T vec4;
  const vec4 x = *reinterpret_cast<const vec4*>(p);
  return f32x4{float(x[0]), float(x[1]), float(x[2]), float(x[3])};
}

template <typename T, int DK, int DV>
__global__ __launch_bounds__(256, (DeltaGradCfg<T, DK, DV>::GROUPS)) void delta_gradients(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ dO,
    const float* __restrict__ s, const float* __restrict__ log_decay, const float* __restrict__ beta,
    const int* __restrict__ lengths, const ChunkRecord* __restrict__ records, const float* __restrict__ errors,
    const float* __restrict__ states, const float* __restrict__ zs, const float* __restrict__ dstates, T* __restrict__ dQ,
    T* __restrict__ dK, T* __restrict__ dV, float* __restrict__ dlog_decay, float* __restrict__ dbeta,
    float* __restrict__ ds_parts, Divisor H, Divisor chunks, int N, float inv_eps, int from_state) {
  using Cfg = DeltaGradCfg<T, DK, DV>;
  using KTile = typename Cfg::KTile;
  using GTile = typename Cfg::GTile;
  using ETile = typename Cfg::ETile;
  using MTile = typename Cfg::MTile;
  constexpr int IN = Cfg::IN, LEVEL = Cfg::LEVEL, NK = Cfg::NK, NTOK = Cfg::NTOK, VS = DV / 32;
  __shared__ __attribute__((aligned(16))) uint16_t room[Cfg::SIZE];
  __shared__ ChunkRecord rec;
  __shared__ __attribute__((aligned(16))) float rq[CHUNK], xv[CHUNK];
  __shared__ float tail[4];
  typedef float Dots[4][CHUNK];
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
    for (int i = tid; i < (hi - lo) * (DK / 4); i += 256) {
      *reinterpret_cast<vec4*>(dQu + size_t(lo) * DK + i * 4) = none;
      *reinterpret_cast<vec4*>(dKu + size_t(lo) * DK + i * 4) = none;
    }
    for (int i = tid; i < (hi - lo) * (DV / 4); i += 256) *reinterpret_cast<vec4*>(dVu + size_t(lo) * DV + i * 4) = none;
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
  RowTile<T, DK, Cfg::PAD> kt, qt;
  {
    using RT = RowTile<T, DV, Cfg::PAD>;
    RT gt, vt;
    gt.fetch(dO + (row_at + row0) * DV, there - row0);
    vt.fetch(V + (row_at + row0) * DV, there - row0);
    kt.fetch(K + (row_at + row0) * DK, there - row0);
    qt.fetch(Q + (row_at + row0) * DK, there - row0);
    if (tid < RECORD_PIECES) reinterpret_cast<u32x4*>(&rec)[tid] = reinterpret_cast<const u32x4*>(records + blockIdx.x)[tid];
    gt.commit(Os);
#pragma unroll
    for (int p = 0; p < RT::PASSES; ++p) {
      const int row = RT::row(p), col = RT::col();
      const size_t at = (size_t(blockIdx.x) * CHUNK + row) * DV + col;
      const f32x4* ep = reinterpret_cast<const f32x4*>(errors + at);
      const f32x4* zp = reinterpret_cast<const f32x4*>(zs + at);
      const f32x4 e0 = ep[0], e1 = ep[1], z0 = zp[0], z1 = zp[1];
      const float b = row0 + row < there ? beta[row_at + row0 + row] : 0.f;
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

  // wave w: key tiles kt0 .. kt0 + NK - 1, token tiles tt0 .. tt0 + NTOK - 1
  const int kt0 = Cfg::KT >= 4 ? w * NK : w % 2, tt0 = Cfg::KT >= 4 ? 0 : w / 2 * 2;
  f32x4 aq[NK][NTOK], ak[NK][NTOK];
  float through = 0.f;   // <D, H>, of the wave's rows
  {
    f32x4 az[NK][NTOK];
#pragma unroll
    for (int x = 0; x < NK; ++x)
#pragma unroll
      for (int t = 0; t < NTOK; ++t) aq[x][t] = ak[x][t] = az[x][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int vs = 0; vs < VS; ++vs) {
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        const size_t at = size_t(blockIdx.x) * DK * DV + size_t(16 * (kt0 + x) + r) * DV + 32 * vs + 8 * q4;
        const f32x4* hp = reinterpret_cast<const f32x4*>(states + at);
        const f32x4* dp = reinterpret_cast<const f32x4*>(dstates + at);
        const f32x4 h0 = hp[0], h1 = hp[1], d0 = dp[0], d1 = dp[1];
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
          aq[x][t] = mm<LEVEL>(hf, gf, aq[x][t]);
          ak[x][t] = mm<LEVEL>(df, ef, ak[x][t]);
          az[x][t] = mm<LEVEL>(hf, zf, az[x][t]);
        }
      }
    }
    // each token's factors; and what the updates of the chunk give to <D, H behind the chunk>
    if (Cfg::KT < 4 && w >= 2) through = 0.f;
    through *= rec.since[CHUNK - 1];
#pragma unroll
    for (int t = 0; t < NTOK; ++t) {
      const int i = 16 * (tt0 + t) + r;
      const float since = rec.since[i], to_end = rec.beta[i] * decay_between(rec.decay[CHUNK - 1], rec.decay[i]);
      float dot = 0.f;
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        f32x4 k = {0.f, 0.f, 0.f, 0.f};
        if (row0 + i < there) k = load_row4(K + (row_at + row0 + i) * DK + 16 * (kt0 + x) + 4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          aq[x][t][v] *= since;
          ak[x][t][v] *= to_end;
          dot = __builtin_fmaf(k[v], ak[x][t][v], dot);
          ak[x][t][v] = __builtin_fmaf(-rec.beta[i] * since, az[x][t][v], ak[x][t][v]);
        }
      }
      through = __builtin_fmaf(rec.rk[i], dot, through);
    }
    through = group_sum<64>(through);
    if (l == 0) tail[w] = through;
  }

  // the masked tiles: rows i of wave w's tile, columns j; lanes hold four columns of a row
  f32x4 pt[4], at[4];
  const int own = 16 * w + r;
  const double g_own = rec.decay[own];
  const float b_own = rec.beta[own];
  {
    bf16x8 gf[VS][IN], zf[VS][LEVEL];
#pragma unroll
    for (int vs = 0; vs < VS; ++vs) {
      GTile::row_frag(Os, own, 32 * vs + 8 * q4, gf[vs]);
      ETile::row_frag(Zs, own, 32 * vs + 8 * q4, zf[vs]);
    }
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      pt[jt] = at[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (jt <= w) {
#pragma unroll
        for (int vs = 0; vs < VS; ++vs) {
          bf16x8 ef[LEVEL];
          ETile::row_frag(Es, 16 * jt + r, 32 * vs + 8 * q4, ef);
          pt[jt] = mm<LEVEL>(ef, gf[vs], pt[jt]);
          at[jt] = mm<LEVEL>(ef, zf[vs], at[jt]);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int j = 16 * jt + 4 * q4 + v;
          const float f = rec.beta[j] * decay_between(g_own, rec.decay[j]);
          pt[jt][v] = j <= own ? pt[jt][v] * f : 0.f;
          at[jt][v] = j < own ? -b_own * at[jt][v] * f : 0.f;
        }
      }
    }
  }
  const float rq_own = rq[own], rk_own = rec.rk[own];
  __syncthreads();   // the rows of dO, E and Z are read
  kt.commit(Ks);
  qt.commit(Qs);
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) {
    const f32x4 k4 = *reinterpret_cast<const f32x4*>(rec.rk + 16 * jt + 4 * q4);
    MTile::store4(Ms, own, 16 * jt + 4 * q4, pt[jt] * k4);
    MTile::store4(Mt, own, 16 * jt + 4 * q4, pt[jt] * (scale * rq_own));
  }
  __syncthreads();
#pragma unroll
  for (int round = 0; round < 2; ++round) {
#pragma unroll
    for (int t = 0; t < NTOK; ++t) {
      const int tt = tt0 + t;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int t0 = 32 * ks + 8 * q4;
        const bool before = 2 * ks <= tt, after = 2 * ks + 1 >= tt;   // columns up to row tt's tile; rows from column tt's tile on
        bf16x8 mf[LEVEL], mt[LEVEL];
        if (before) MTile::row_frag(Ms, 16 * tt + r, t0, mf);
        if (after) MTile::col_frag(Mt, t0, t0 + 4, 16 * tt, r, mt);
#pragma unroll
        for (int x = 0; x < NK; ++x) {
          bf16x8 kf[IN];
          KTile::col_frag(Ks, t0, t0 + 4, 16 * (kt0 + x), r, kf);
          if (round == 0) {
            bf16x8 qf[IN];
            if (before) aq[x][t] = mm<LEVEL>(kf, mf, aq[x][t]);
            if (after) {
              KTile::col_frag(Qs, t0, t0 + 4, 16 * (kt0 + x), r, qf);
              ak[x][t] = mm<LEVEL>(qf, mt, ak[x][t]);
            }
          } else {
            if (before) ak[x][t] = mm<LEVEL>(kf, mf, ak[x][t]);
            if (after) ak[x][t] = mm<LEVEL>(kf, mt, ak[x][t]);
          }
        }
      }
    }
    if (round == 0) {
      __syncthreads();
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) {
        const f32x4 k4 = *reinterpret_cast<const f32x4*>(rec.rk + 16 * jt + 4 * q4);
        MTile::store4(Ms, own, 16 * jt + 4 * q4, at[jt] * k4);
        MTile::store4(Mt, own, 16 * jt + 4 * q4, at[jt] * rk_own);
      }
      __syncthreads();
    }
  }

  __syncthreads();
  // through the normalisation: dq = (dqh - qh (qh . dqh)) / |q|; a row below eps was divided by eps alone
#pragma unroll
  for (int t = 0; t < NTOK; ++t) {
    const int i = 16 * (tt0 + t) + r;
    float dq = 0.f, dk = 0.f;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      f32x4 q = {0.f, 0.f, 0.f, 0.f}, k = q;
      if (row0 + i < there) {
        q = load_row4(Q + (row_at + row0 + i) * DK + 16 * (kt0 + x) + 4 * q4);
        k = load_row4(K + (row_at + row0 + i) * DK + 16 * (kt0 + x) + 4 * q4);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        dq = __builtin_fmaf(q[v], aq[x][t][v], dq);
        dk = __builtin_fmaf(k[v], ak[x][t][v], dk);
      }
    }
    dq += __shfl_xor(dq, 16, 64);
    dk += __shfl_xor(dk, 16, 64);
    dq += __shfl_xor(dq, 32, 64);
    dk += __shfl_xor(dk, 32, 64);
    if (q4 == 0) {
      qdot[Cfg::KT >= 4 ? w : w % 2][i] = dq;
      kdot[Cfg::KT >= 4 ? w : w % 2][i] = dk;
    }
  }
  __syncthreads();
  constexpr int SHARES = Cfg::KT >= 4 ? 4 : 2;
#pragma unroll
  for (int t = 0; t < NTOK; ++t) {
    const int i = 16 * (tt0 + t) + r;
    float dq = 0.f, dk = 0.f;
#pragma unroll
    for (int n = 0; n < SHARES; ++n) {
      dq += qdot[n][i];
      dk += kdot[n][i];
    }
    const float fq = rq[i], fk = rec.rk[i];
    const float cq = fq == inv_eps ? 0.f : fq * (fq * dq), ck = fk == inv_eps ? 0.f : fk * (fk * dk);
    if (row0 + i < there) {
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        const size_t at_ = size_t(row0 + i) * DK + 16 * (kt0 + x) + 4 * q4;
        const f32x4 q = load_row4(Q + row_at * DK + at_), k = load_row4(K + row_at * DK + at_);
        typedef __attribute__((ext_vector_type(4))) T vec4;
        vec4 gq, gk;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          gq[v] = T(scale * (fq * __builtin_fmaf(-cq, q[v], aq[x][t][v])));
          gk[v] = T(fk * __builtin_fmaf(-ck, k[v], ak[x][t][v]));
        }
        *reinterpret_cast<vec4*>(dQu + at_) = gq;
        *reinterpret_cast<vec4*>(dKu + at_) = gk;
      }
    }
  }
  if (w == 0) {   // lane l: token l
    float dot = 0.f;
#pragma unroll
    for (int n = 0; n < SHARES; ++n) dot += qdot[n][l];
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
      flow += double(tail[0]) + double(tail[1]) + double(tail[2]) + double(tail[3]);
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

template <typename T, int DK>
hipError_t run_rev(const DeltaArgs& a) {
  constexpr int VC = sizeof(T) == 4 && DK == 128 ? 16 : 32;   // (what the LDS holds)
  const int units = a.B * a.H, parts = a.dv / VC;
  return launch_kernel("delta_rev_scan", delta_rev_scan<T, DK, VC>, dim3(unsigned(units * parts)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.dO), a.s, a.seq_len,
                       a.dstate, a.dstate_in, static_cast<const ChunkRecord*>(a.records), a.w_cols, a.zs, a.dstates, Divisor(a.H),
                       Divisor(parts), a.N, units, a.dv, 1.0f / a.eps);
}

template <typename T, int DK, int DV>
hipError_t run_gradients(const DeltaArgs& a) {
  const int chunks = delta_chunks(a.N);
  return launch_kernel("delta_gradients", delta_gradients<T, DK, DV>, dim3(unsigned(a.B * a.H * chunks)), dim3(256), 0, a.stream,
                       static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.V),
                       static_cast<const T*>(a.dO), a.s, a.log_decay, a.beta, a.seq_len,
                       static_cast<const ChunkRecord*>(a.records), a.errors, a.states, a.zs,
                       a.dstates, static_cast<T*>(a.dQ), static_cast<T*>(a.dK), static_cast<T*>(a.dV), a.dlog_decay, a.dbeta,
                       a.ds_parts, Divisor(a.H), Divisor(chunks), a.N, 1.0f / a.eps, int(a.state_in != nullptr));
}

template <typename T, int DK>
hipError_t run_backward(const DeltaArgs& a) {
  hipError_t err = run_rev<T, DK>(a);
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
