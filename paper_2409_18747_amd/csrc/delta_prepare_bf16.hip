// The gated delta rule: what a chunk's rows of K and its gates come to by themselves (delta.h).  All chunks at once, a
// workgroup each: the decays and the rows' factors (ChunkRecord), and the 64 x 64 matrix W as the operand fragments that the
// scans read, once by rows and, for a backward, once more by columns (18 KB each).
//   A workgroup is one dependent chain - rows, A, the diagonal blocks, two sizes of blocks below them - of some 20000 cycles, so
// that what counts is how many a compute unit holds: the matrix takes the rows' place in the LDS and steps of the blocks its empty
// quarter, 20 KB in all, and a diagonal block takes four registers to a lane, not 32.  16 heads of 32768 rows of 64 with a backward
// take 73 us, the rate of a copy; 32 x 16 heads of 2048 rows of 128 without 118 us, 4.0 TB/s (three to a unit and a column of a
// block to a lane: 101 and 205 us).
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

// acc - A diag(f) B for 16 x 16 blocks on the fp32 matrix instruction, A's and B's element (0, 0) at a and b.
constexpr int WP = CHUNK + 4;   // pitch of the fp32 matrices
__device__ __forceinline__ f32x4 block_product(const float* a, const float* f, const float* b, f32x4 acc, int r, int q4) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int at = 4 * k + q4;
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(-a[r * WP + at] * f[at], b[at * WP + r], acc, 0, 0, 0);
  }
  return acc;
}
__device__ __forceinline__ f32x4 load_block(const float* a, int r, int q4) {
  f32x4 x;
#pragma unroll
  for (int v = 0; v < 4; ++v) x[v] = a[(4 * q4 + v) * WP + r];
  return x;
}
__device__ __forceinline__ void store_block(float* a, f32x4 x, int r, int q4) {
#pragma unroll
  for (int v = 0; v < 4; ++v) a[(4 * q4 + v) * WP + r] = x[v];
}

// The sum of the lanes r, 16 + r, 32 + r and 48 + r, in all of them.  (Two registers to a swap: of one the compiler takes the two
// results for the same.)
__device__ __forceinline__ float over_quarters(float x) {
  unsigned a = __builtin_bit_cast(unsigned, x), b = a;
  asm("" : "+v"(b));
  const auto pairs = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = b = __builtin_bit_cast(unsigned, __builtin_bit_cast(float, unsigned(pairs[0])) + __builtin_bit_cast(float, unsigned(pairs[1])));
  asm("" : "+v"(b));
  const auto halves = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return __builtin_bit_cast(float, unsigned(halves[0])) + __builtin_bit_cast(float, unsigned(halves[1]));
}

// W takes A's place block by block.  Within a diagonal block of 16 it is found row by row, W_i = A_i - sum over j < i of A_ij b_j
// W_j, so that no power of A, which may be large, is formed; W of two neighbouring diagonal blocks then gives the block below
// them, W21 = (I - W22 b2) A21 (I - b1 W11), of 16 and then of 32.
template <typename T, int DK>
struct DeltaPrepareCfg {
  using Tile = PartTile<CHUNK, DK, Rows<T>::PARTS>;
  static constexpr int ROOM = 2 * Tile::SIZE > 4 * CHUNK * WP ? 2 * Tile::SIZE : 4 * CHUNK * WP;
  static constexpr int LDS_BYTES = ROOM + int(sizeof(ChunkRecord));
  static constexpr int AT_ONCE = 160 * 1024 / LDS_BYTES < 8 ? 160 * 1024 / LDS_BYTES : 8;   // workgroups to a compute unit
};

template <typename T, int DK>
__global__ __launch_bounds__(256, (DeltaPrepareCfg<T, DK>::AT_ONCE)) void delta_prepare(const T* __restrict__ K, const float* __restrict__ log_decay,
                                                        const float* __restrict__ beta, const int* __restrict__ lengths,
                                                        ChunkRecord* __restrict__ records, uint16_t* __restrict__ w_rows,
                                                        uint16_t* __restrict__ w_cols, Divisor H, Divisor chunks, int N,
                                                        float inv_eps) {
  using Tile = PartTile<CHUNK, DK, Rows<T>::PARTS>;
  __shared__ __attribute__((aligned(16))) char room[DeltaPrepareCfg<T, DK>::ROOM];   // the rows, then As
  __shared__ ChunkRecord rec;
  uint16_t* const Ks = reinterpret_cast<uint16_t*>(room);
  float* const As = reinterpret_cast<float*>(room);
  float* const Xs = As + 32;   // the upper right quarter, which is no one's: the diagonal blocks times b, then a step of the blocks below
  const int unit = quotient(blockIdx.x, chunks), c = blockIdx.x - unit * chunks.n, row0 = c * CHUNK;
  const int there = valid_rows(lengths, unit, H, N);
  if (row0 >= there) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  RowTile<T, DK> kt;
  kt.fetch(K + (size_t(unit) * N + row0) * DK, there - row0);
  float* const diagonal = Xs + 16 * (w / 2) * WP + 16 * (w % 2);
  double g = 0.0;
  if (w == 0) {
    const bool here = row0 + l < there;
    const size_t at = size_t(unit) * N + row0 + l;
    g = here && log_decay != nullptr ? log2_decay(log_decay[at]) : 0.0;
    rec.beta[l] = here ? beta[at] : 0.f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double before = __shfl_up(g, d, 64);
      if (l >= d) g += before;
    }
    rec.decay[l] = g;
  }
  kt.commit(Ks);
  kt.store_factors(rec.rk, inv_eps);
  __syncthreads();
  if (w == 0) {
    const float rk = rec.rk[l], since = decay_between(g, 0.0);
    rec.rk_to_tile[l] = rk * decay_between(rec.decay[l | 15], g);
    rec.rk_to_end[l] = rk * decay_between(rec.decay[CHUNK - 1], g);
    rec.rk_since[l] = rk * since;
    rec.since[l] = since;
    rec.in_tile[l] = decay_between(g, l < 16 ? 0.0 : rec.decay[l / 16 * 16 - 1]);
    if (l < 16) rec.between[l / 4][l % 4] = l / 4 > l % 4 ? decay_between(rec.decay[l / 4 * 16 - 1], rec.decay[l % 4 * 16 + 15]) : 0.f;
    if (l == 0) {
      state_factor(rec.decay[CHUNK - 1], rec.times, rec.plus);
      rec.unused[0] = rec.unused[1] = 0.f;
    }
  }
  {
    bf16x8 own[DK / 32][Rows<T>::PARTS];
#pragma unroll
    for (int ks = 0; ks < DK / 32; ++ks) Tile::row_frag(Ks, 16 * w + r, 32 * ks + 8 * q4, own[ks]);
    f32x4 tiles[4];
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
      if (jt <= w) {
#pragma unroll
        for (int ks = 0; ks < DK / 32; ++ks) {
          bf16x8 other[Rows<T>::PARTS];
          Tile::row_frag(Ks, 16 * jt + r, 32 * ks + 8 * q4, other);
          t = mm<3>(own[ks], other, t);
        }
        const int j = 16 * jt + r;
        const float rj = rec.rk[j];
        const double gj = rec.decay[j];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int i = 16 * w + 4 * q4 + v;
          t[v] = j < i ? t[v] * rec.rk[i] * rj * decay_between(rec.decay[i], gj) : 0.f;
        }
      }
      tiles[jt] = t;
    }
    __syncthreads();   // the rows are read
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      if (jt == w) store_block(diagonal, tiles[jt] * rec.beta[16 * jt + r], r, q4);
      if (jt <= (w | 1)) store_block(As + 16 * w * WP + 16 * jt, tiles[jt], r, q4);   // (what the fragments hold of the tiles above: zeros)
    }
  }
  wave_lds_sync();
  {   // the diagonal blocks, one to a wave: a lane has every fourth row of a column, and a row is found from the sums of four lanes
    float* a = As + 16 * w * WP + 16 * w;
    float x[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = a[(4 * t + q4) * WP + r];   // (0 from the diagonal on; so is `diagonal`, where x is not found yet)
#pragma unroll
    for (int i = 2; i < 16; ++i) {
      float sum = 0.f;
#pragma unroll
      for (int t = 0; 4 * t < i; ++t) sum = __builtin_fmaf(-diagonal[i * WP + 4 * t + q4], x[t], sum);
      sum = over_quarters(sum);
      x[i / 4] += q4 == i % 4 ? sum : 0.f;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) a[(4 * t + q4) * WP + r] = x[t];
  }
  __syncthreads();
  if (w < 2) {   // blocks (1, 0) and (3, 2)
    const int i0 = 32 * w + 16, j0 = 32 * w;
    float* a = As + i0 * WP + j0;
    f32x4 x = block_product(a, rec.beta + j0, As + j0 * WP + j0, load_block(a, r, q4), r, q4);
    store_block(Xs + 16 * w * WP, x, r, q4);
    wave_lds_sync();
    x = block_product(As + i0 * WP + i0, rec.beta + i0, Xs + 16 * w * WP, x, r, q4);
    store_block(a, x, r, q4);
  }
  __syncthreads();
  {   // the lower left 32 x 32, a block to a wave
    const int bi = w / 2, bj = w % 2, i0 = 32 + 16 * bi, j0 = 16 * bj;
    f32x4 x = load_block(As + i0 * WP + j0, r, q4);
    for (int bk = bj; bk < 2; ++bk)
      x = block_product(As + i0 * WP + 16 * bk, rec.beta + 16 * bk, As + 16 * bk * WP + j0, x, r, q4);
    store_block(Xs + 16 * bi * WP + j0, x, r, q4);
    __syncthreads();
    for (int bk = 0; bk <= bi; ++bk)
      x = block_product(As + i0 * WP + 32 + 16 * bk, rec.beta + 32 + 16 * bk, Xs + 16 * bk * WP + j0, x, r, q4);
    store_block(As + i0 * WP + j0, x, r, q4);
  }
  __syncthreads();
  if (tid < RECORD_PIECES)
    reinterpret_cast<u32x4*>(records + blockIdx.x)[tid] = reinterpret_cast<const u32x4*>(&rec)[tid];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    bf16x8 f[3];
    if (w_row_there(w, ks)) {
      // W b: its columns take the factors of the rows that they are multiplied by
      const float* from = As + (16 * w + r) * WP + 32 * ks + 4 * q4;
      const float* b = rec.beta + 32 * ks + 4 * q4;
      split8<3>(*reinterpret_cast<const f32x4*>(from) * *reinterpret_cast<const f32x4*>(b),
                *reinterpret_cast<const f32x4*>(from + 16) * *reinterpret_cast<const f32x4*>(b + 16), f);
      uint16_t* to = w_rows + size_t(blockIdx.x) * W_ELEMS + w_row_frag(w, ks) * 3 * 512 + l * 8;
#pragma unroll
      for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4*>(to + i * 512) = __builtin_bit_cast(u32x4, f[i]);
    }
    if (w_cols != nullptr && w_col_there(w, ks)) {
      const float* from = As + (32 * ks + 4 * q4) * WP + 16 * w + r;
      f32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = from[i * WP];
        hi[i] = from[(16 + i) * WP];
      }
      split8<3>(lo, hi, f);
      uint16_t* to = w_cols + size_t(blockIdx.x) * W_ELEMS + w_col_frag(w, ks) * 3 * 512 + l * 8;
#pragma unroll
      for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4*>(to + i * 512) = __builtin_bit_cast(u32x4, f[i]);
    }
  }
}

}  // namespace

hipError_t DELTA_SYM(delta_prepare)(const DeltaArgs& a) {
  typedef DELTA_T T;
  const int chunks = delta_chunks(a.N);
  const auto run = [&](auto kernel) {
    return launch_kernel("delta_prepare", kernel, dim3(unsigned(a.B * a.H * chunks)), dim3(256), 0, a.stream,
                         static_cast<const T*>(a.K), a.log_decay, a.beta, a.seq_len, static_cast<ChunkRecord*>(a.records), a.w_rows,
                         a.w_cols, Divisor(a.H), Divisor(chunks), a.N, largest_factor(a.eps));
  };
  return a.dk == 32 ? run(delta_prepare<T, 32>) : a.dk == 64 ? run(delta_prepare<T, 64>) : run(delta_prepare<T, 128>);
}

}  // namespace cottn
