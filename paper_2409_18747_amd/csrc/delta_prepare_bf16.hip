// The gated delta rule: what a chunk's rows of K and its gates come to by themselves (delta.h).  All chunks at once, a
// workgroup each: the rows' factors 1 / norm, the decays from the chunk's start, and the 64 x 64 matrix W.
#include "device_common.h"
#include "delta.h"
#include "delta_elem.h"

namespace cottn {
namespace {

// fp32 products of 16 x 16 blocks on the fp32 matrix instruction: acc +- A diag(f) B, A's and B's element (0, 0) at a and b.
constexpr int WP = CHUNK + 4;   // pitch of the fp32 matrices
__device__ __forceinline__ f32x4 block_product(const float* a, int pa, const float* f, const float* b, int pb, f32x4 acc, int r, int q4) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int at = 4 * k + q4;
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(-a[r * pa + at] * f[at], b[at * pb + r], acc, 0, 0, 0);
  }
  return acc;
}
__device__ __forceinline__ f32x4 load_block(const float* a, int pitch, int r, int q4) {
  f32x4 x;
#pragma unroll
  for (int v = 0; v < 4; ++v) x[v] = a[(4 * q4 + v) * pitch + r];
  return x;
}
__device__ __forceinline__ void store_block(float* a, int pitch, f32x4 x, int r, int q4) {
#pragma unroll
  for (int v = 0; v < 4; ++v) a[(4 * q4 + v) * pitch + r] = x[v];
}

// W of two neighbouring diagonal blocks gives the block below them: W21 = (I - W22 b2) A21 (I - b1 W11).  Within a block of 16
// it is found row by row, W_i = A_i - sum over j < i of A_ij b_j W_j, so that no power of A, which may be large, is formed.
template <typename T, int DK>
__global__ __launch_bounds__(256) void delta_prepare(const T* __restrict__ K, const float* __restrict__ log_decay,
                                                     const float* __restrict__ beta, const int* __restrict__ lengths,
                                                     float* __restrict__ W, double* __restrict__ decays,
                                                     float* __restrict__ factors, Divisor H, Divisor chunks, int N, float eps) {
  using Tile = PartTile<CHUNK, DK, Rows<T>::PARTS>;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[Tile::SIZE];
  __shared__ __attribute__((aligned(16))) float As[CHUNK * WP], Ws[CHUNK * WP], Xs[32 * WP];
  __shared__ double Gs[CHUNK];
  __shared__ __attribute__((aligned(16))) float rk[CHUNK], bs[CHUNK];
  const int unit = quotient(blockIdx.x, chunks), c = blockIdx.x - unit * chunks.n, row0 = c * CHUNK;
  const int there = valid_rows(lengths, unit, H, N);
  if (row0 >= there) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, r = l % 16, q4 = l / 16;
  RowTile<T, DK> kt;
  kt.fetch(K + size_t(unit) * N * DK, row0, there);
  if (w == 0) {
    const bool here = row0 + l < there;
    const size_t at = size_t(unit) * N + row0 + l;
    double g = here && log_decay != nullptr ? log2_decay(log_decay[at]) : 0.0;
    bs[l] = here ? beta[at] : 0.f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double before = __shfl_up(g, d, 64);
      if (l >= d) g += before;
    }
    Gs[l] = g;
    decays[size_t(blockIdx.x) * CHUNK + l] = g;
  }
  kt.commit(Ks);
  kt.store_factors(rk, eps);
  for (int i = tid; i < CHUNK * WP; i += 256) Ws[i] = 0.f;
  __syncthreads();
  if (tid < CHUNK) factors[size_t(blockIdx.x) * CHUNK + tid] = rk[tid];
  {
    bf16x8 own[DK / 32][Rows<T>::PARTS];
#pragma unroll
    for (int ks = 0; ks < DK / 32; ++ks) Tile::row_frag(Ks, 16 * w + r, 32 * ks + 8 * q4, own[ks]);
    for (int jt = 0; jt <= w; ++jt) {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < DK / 32; ++ks) {
        bf16x8 other[Rows<T>::PARTS];
        Tile::row_frag(Ks, 16 * jt + r, 32 * ks + 8 * q4, other);
        t = mm<3>(own[ks], other, t);
      }
      const int j = 16 * jt + r;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int i = 16 * w + 4 * q4 + v;
        As[i * WP + j] = j < i ? t[v] * rk[i] * rk[j] * decay_between(Gs[i], Gs[j]) : 0.f;
      }
    }
  }
  wave_lds_sync();
  {   // the diagonal blocks, one to a wave: a lane finds a column
    const float* a = As + 16 * w * WP + 16 * w;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float sum = a[i * WP + r];
#pragma unroll
      for (int j = 1; j < i; ++j) sum = __builtin_fmaf(-a[i * WP + j] * bs[16 * w + j], x[j], sum);
      x[i] = r < i ? sum : 0.f;
      if (q4 == 0) Ws[(16 * w + i) * WP + 16 * w + r] = x[i];
    }
  }
  __syncthreads();
  if (w < 2) {   // blocks (1, 0) and (3, 2)
    const int i0 = 32 * w + 16, j0 = 32 * w;
    f32x4 x = block_product(As + i0 * WP + j0, WP, bs + j0, Ws + j0 * WP + j0, WP, load_block(As + i0 * WP + j0, WP, r, q4), r, q4);
    store_block(Xs + 16 * w * WP, WP, x, r, q4);
    wave_lds_sync();
    x = block_product(Ws + i0 * WP + i0, WP, bs + i0, Xs + 16 * w * WP, WP, x, r, q4);
    store_block(Ws + i0 * WP + j0, WP, x, r, q4);
  }
  __syncthreads();
  {   // the lower left 32 x 32, a block to a wave
    const int bi = w / 2, bj = w % 2, i0 = 32 + 16 * bi, j0 = 16 * bj;
    f32x4 x = load_block(As + i0 * WP + j0, WP, r, q4);
    for (int bk = bj; bk < 2; ++bk)
      x = block_product(As + i0 * WP + 16 * bk, WP, bs + 16 * bk, Ws + 16 * bk * WP + j0, WP, x, r, q4);
    store_block(Xs + 16 * bi * WP + j0, WP, x, r, q4);
    __syncthreads();
    for (int bk = 0; bk <= bi; ++bk)
      x = block_product(Ws + i0 * WP + 32 + 16 * bk, WP, bs + 32 + 16 * bk, Xs + 16 * bk * WP + j0, WP, x, r, q4);
    store_block(Ws + i0 * WP + j0, WP, x, r, q4);
  }
  __syncthreads();
  float* out = W + size_t(blockIdx.x) * CHUNK * CHUNK;
#pragma unroll
  for (int i = 0; i < CHUNK * CHUNK / 4 / 256; ++i) {
    const int at = i * 256 + tid, row = at / 16, col = at % 16 * 4;
    reinterpret_cast<f32x4*>(out)[at] = *reinterpret_cast<const f32x4*>(Ws + row * WP + col);
  }
}

}  // namespace

hipError_t DELTA_SYM(delta_prepare)(const DeltaArgs& a) {
  typedef DELTA_T T;
  const int chunks = delta_chunks(a.N);
  const auto run = [&](auto kernel) {
    return launch_kernel("delta_prepare", kernel, dim3(unsigned(a.B * a.H * chunks)), dim3(256), 0, a.stream,
                         static_cast<const T*>(a.K), a.log_decay, a.beta, a.seq_len, a.W, a.decays, a.factors, Divisor(a.H),
                         Divisor(chunks), a.N, a.eps);
  };
  return a.dk == 32 ? run(delta_prepare<T, 32>) : a.dk == 64 ? run(delta_prepare<T, 64>) : run(delta_prepare<T, 128>);
}

}  // namespace cottn
