// What the kernels of the gated delta rule share.  With qh, kh the normalised rows, g_t = exp(log_decay_t) and b_t = beta_t
//     H_t = g_t (I - b_t kh_t^T kh_t) H_(t-1) + b_t kh_t^T v_t,    o_t = s qh_t H_t.
//
// A chunk takes 64 rows; G_i is the product of the decays from its first row to row i, H the state before it and
//     A_ij = (G_i / G_j) kh_i . kh_j  for j < i, else 0,      P_ij = (G_i / G_j) qh_i . kh_j  for j <= i, else 0,
//     W = A (I + b A)^-1, strictly lower: what row j's value leaves in row i's prediction after the rows between took theirs
// With the rows' factors b as diagonal matrices and D the gradient with respect to the state behind the chunk:
//     Y = V - G Kh H,  E = Y - W b Y,  U = b E,  O = s (G Qh H + P U),  H <- G_n H + (G_n/G Kh)^T U
//     dO' = s dO,  F = P^T dO' + (G_n/G) Kh D,  Z = F - W^T b F,  X = b Z,  D <- G_n D + (G Qh)^T dO' - (G Kh)^T X
//     dV = X,  db_i = z_i . e_i,  p_ij = (G_i/G_j) dO'_i . u_j (j <= i),  a_ij = -(G_i/G_j) x_i . u_j (j < i)
//     dQh = G dO' H^T + p Kh,   dKh = (G_n/G) U D^T - G X H^T + p^T Qh + (a + a^T) Kh
//     d log g_t = <D, H behind the chunk> + sum over i >= t of (qh_i . dqh_i - x_i . v_i),   ds = sum of qh_i . dqh_i / s
// (E is the error of a row's prediction; neither b nor a decay is ever divided by.)  W's entries are products of rows with
// contractions, at most 1 in magnitude for 0 <= b <= 2.  Every decay that is formed has an exponent that is not positive.
//
// Precision.  Products take bfloat16 parts of their operands, each part the rest that rounding the ones before left over:
// bfloat16 rows are one part, fp16 rows two and fp32 rows three, exactly; what is computed takes three, and of the products of
// parts those i + j < LEVEL are formed: LEVEL 3 leaves out less than 2^-24 of a product, LEVEL 2 less than 2^-15.  All takes 3 but
// for the last products of a forward in 16 bits, of rows with the state and of P with U, whose operands are in two parts (H, P and
// U): nothing goes on from there, and an element has met one rounding that counts, its own (bf16 2^-8, fp16 2^-11).  32 heads of 500
// rows of 128 in bf16 are 1.65803e-3 from 64 bits, the exact results rounded 1.65802e-3; in fp16, of 64, 2.0756e-4 and 2.0750e-4.
// With three parts prompts of 32 x 16 heads of 2048 rows of 128 take 689 us in the scan, not 609, and fp16 has no room for them.
//
// Included behind device_common.h.
#pragma once

namespace cottn {
namespace {

using namespace COTTN_NS;

constexpr int CHUNK = 64;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

template <typename T> struct Rows;
template <> struct Rows<__bf16> { static constexpr int PARTS = 1; };
template <> struct Rows<_Float16> { static constexpr int PARTS = 2; };
template <> struct Rows<float> { static constexpr int PARTS = 3; };
// parts of operands that only enter a forward's results in the rows' type
template <typename T> constexpr int RESULT_LEVEL = sizeof(T) == 4 ? 3 : 2;

// Four values as N parts, two to a word.
template <int N>
__device__ __forceinline__ void split4(f32x4 x, uint2 (&parts)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    parts[i] = uint2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    if (i + 1 < N) {
      float p[4];
      unpack2(parts[i].x, p[0], p[1]);
      unpack2(parts[i].y, p[2], p[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] -= p[e];
    }
  }
}
template <int N>
__device__ __forceinline__ void split8(f32x4 lo, f32x4 hi, bf16x8 (&parts)[N]) {
  uint2 a[N], b[N];
  split4<N>(lo, a);
  split4<N>(hi, b);
#pragma unroll
  for (int i = 0; i < N; ++i) parts[i] = __builtin_bit_cast(bf16x8, u32x4{a[i].x, a[i].y, b[i].x, b[i].y});
}

// The values that parts stand for.
template <int N>
__device__ __forceinline__ void join8(const bf16x8 (&parts)[N], f32x4& lo, f32x4& hi) {
  lo = hi = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = N - 1; i >= 0; --i) {
    const u32x4 w = __builtin_bit_cast(u32x4, parts[i]);
    float a, b;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      unpack2(w[e], a, b);
      lo[2 * e] += a;
      lo[2 * e + 1] += b;
      unpack2(w[2 + e], a, b);
      hi[2 * e] += a;
      hi[2 * e + 1] += b;
    }
  }
}

// acc (16 x 16) += a (16 x 32) b (32 x 16), the smallest products of parts first.
template <int LEVEL, int NA, int NB>
__device__ __forceinline__ f32x4 mm(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 acc) {
#pragma unroll
  for (int sum = LEVEL - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = sum - i;
      if (j >= 0 && j < NB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc, 0, 0, 0);
    }
  return acc;
}

// The same for N tiles with an operand in common, product by product: neighbouring matrix instructions do not wait for each other.
template <int LEVEL, int N, int NA, int NB>
__device__ __forceinline__ void mm_each(const bf16x8 (&a)[N][NA], const bf16x8 (&b)[NB], f32x4* acc) {
#pragma unroll
  for (int sum = LEVEL - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = sum - i;
      if (j >= 0 && j < NB) {
#pragma unroll
        for (int t = 0; t < N; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t][i], b[j], acc[t], 0, 0, 0);
      }
    }
}
template <int LEVEL, int N, int NA, int NB>
__device__ __forceinline__ void mm_each(const bf16x8 (&a)[NA], const bf16x8 (&b)[N][NB], f32x4* acc) {
#pragma unroll
  for (int sum = LEVEL - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = sum - i;
      if (j >= 0 && j < NB) {
#pragma unroll
        for (int t = 0; t < N; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[t][j], acc[t], 0, 0, 0);
      }
    }
}

// Eight consecutive elements of a row as they lie in memory, as fp32 and as parts.
template <typename T>
struct Raw8 {
  static constexpr int PIECES = sizeof(T) / 2, PARTS = Rows<T>::PARTS;
  u32x4 w[PIECES];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
  }
  __device__ __forceinline__ void values(f32x4& lo, f32x4& hi) const {
    if constexpr (sizeof(T) == 4) {
      lo = __builtin_bit_cast(f32x4, w[0]);
      hi = __builtin_bit_cast(f32x4, w[PIECES - 1]);
    } else {
      typedef __attribute__((ext_vector_type(8))) T vec8;
      const vec8 x = __builtin_bit_cast(vec8, w[0]);
      lo = f32x4{float(x[0]), float(x[1]), float(x[2]), float(x[3])};
      hi = f32x4{float(x[4]), float(x[5]), float(x[6]), float(x[7])};
    }
  }
  __device__ __forceinline__ void parts(bf16x8 (&p)[PARTS]) const {
    if constexpr (PARTS == 1) {
      p[0] = __builtin_bit_cast(bf16x8, w[0]);
    } else {
      f32x4 lo, hi;
      values(lo, hi);
      split8<PARTS>(lo, hi, p);
    }
  }
  __device__ __forceinline__ float sum_sq() const {
    if constexpr (PARTS == 1) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) s = dot2_self(w[0][i], s);
      return s;
    }
    f32x4 lo, hi;
    values(lo, hi);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_fmaf(lo[i], lo[i], __builtin_fmaf(hi[i], hi[i], s));
    return s;
  }
};

// Slots of operand fragments.  Lane row q = lane / 16 of a fragment of 32 k indices has the slots 8 q .. 8 q + 7 where it is read
// from rows in LDS or memory, and 4 q .. 4 q + 3 and 16 + 4 q .. 16 + 4 q + 3 where it is two accumulator tiles side by side (or
// is to meet one that is): those tiles become operands without leaving their lanes.

// A tile of 16-bit parts in LDS: plane after plane of ROWS rows, each PITCH wide.  (Rows 16 apart from a multiple of 32 are read
// fastest, device_common.h; 8 where the LDS has no room for that.)
template <int ROWS, int COLS, int PARTS, int PAD = 16>
struct PartTile {
  static constexpr int PITCH = COLS + PAD, PLANE = ROWS * PITCH, SIZE = PARTS * PLANE;
  // operand fragment whose k slots are columns c .. c + 7 of a row
  template <int N = PARTS>
  static __device__ __forceinline__ void row_frag(const uint16_t* tile, int row, int c, bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(tile + i * PLANE + row * PITCH + c));
  }
  // operand fragment whose k slots are rows r0 .. r0 + 3 and r1 .. r1 + 3 of column col0 + r
  template <int N = PARTS>
  static __device__ __forceinline__ void col_frag(const uint16_t* tile, int r0, int r1, int col0, int r, bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = __builtin_bit_cast(bf16x8, lds_col_frag(tile + i * PLANE, PITCH, r0, r1, col0, r));
  }
  // the same of 16 columns that are four from `first` on, four from first + 8 on and so forth: lane r has first + 8 (r / 4) + r % 4
  template <int N = PARTS>
  static __device__ __forceinline__ void spread_col_frag(const uint16_t* tile, int r0, int r1, int first, int r, bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint16_t* p = tile + i * PLANE + (r >> 2) * PITCH + first + 8 * (r & 3);
      const s16x4 lo = lds_read_tr(p + r0 * PITCH), hi = lds_read_tr(p + r1 * PITCH);
      f[i] = __builtin_bit_cast(bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
  }
  // columns c .. c + 3 of a row as fp32
  static __device__ __forceinline__ f32x4 row4(const uint16_t* tile, int row, int c) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = PARTS - 1; i >= 0; --i) {
      const uint2 w = *reinterpret_cast<const uint2*>(tile + i * PLANE + row * PITCH + c);
      float t[4];
      unpack2(w.x, t[0], t[1]);
      unpack2(w.y, t[2], t[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += t[e];
    }
    return x;
  }
  // rows row0 .. row0 + 3 of column col0 + r as fp32
  static __device__ __forceinline__ f32x4 col4(const uint16_t* tile, int row0, int col0, int r) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = PARTS - 1; i >= 0; --i) {
      const uint2 w = __builtin_bit_cast(uint2, lds_read_tr(tile + i * PLANE + (row0 + (r >> 2)) * PITCH + col0 + (r & 3) * 4));
      float t[4];
      unpack2(w.x, t[0], t[1]);
      unpack2(w.y, t[2], t[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += t[e];
    }
    return x;
  }
  template <int N = PARTS>
  static __device__ __forceinline__ void store4(uint16_t* tile, int row, int c, f32x4 x) {
    uint2 p[N];
    split4<N>(x, p);
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<uint2*>(tile + i * PLANE + row * PITCH + c) = p[i];
  }
  template <int N>
  static __device__ __forceinline__ void store8(uint16_t* tile, int row, int c, const bf16x8 (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(tile + i * PLANE + row * PITCH + c) = __builtin_bit_cast(u32x4, p[i]);
  }
};

// Factors of rows are 2^75 at most: no sum of squares but 0 gives more (2^74.5), and 0 is what a row of zeros times any is; a value
// times 1 / eps may leave fp32, and infinity times a zero row is not 0.  The product of two rows takes their factors one after the
// other, for the same reason.  Gradients with respect to rows below eps are over eps itself.
constexpr float LARGEST_FACTOR = 0x1p75f;
inline float largest_factor(float eps) { return fminf(1.0f / eps, LARGEST_FACTOR); }
inline float over_eps(float eps) { return fminf(1.0f / eps, 0x1.fffffep127f); }
// 1 / max(norm, eps) of a row from its sum of squares, to a unit of fp32: the reciprocal square root instruction, which takes what is
// below the normal numbers for 0.  (8192 rows of one feature come out 0.60 of 2^-24 from 1 in the root mean square, with a Newton step
// 0.52.)
__device__ __forceinline__ float row_factor(float sum_sq, float inv_eps) {
  const bool tiny = sum_sq < 0x1p-126f;
  const float y = __builtin_amdgcn_rsqf(tiny ? 0x1p64f * sum_sq : sum_sq);
  return fminf(tiny ? 0x1p32f * y : y, inv_eps);
}

// 64 rows of D elements on their way from memory to LDS: D / 8 neighbouring lanes share a row.
template <typename T, int D, int PAD = 16, int THREADS = 256>
struct RowTile {
  static constexpr int LPR = D / 8, RPP = THREADS / LPR, PASSES = RPP < CHUNK ? CHUNK / RPP : 1, PARTS = Rows<T>::PARTS;
  using Tile = PartTile<CHUNK, D, PARTS, PAD>;
  Raw8<T> raw[PASSES];
  static __device__ __forceinline__ int thread() { return int(threadIdx.x) % THREADS; }   // (of one half of a workgroup's waves)
  static __device__ __forceinline__ int row(int p) { return p * RPP + thread() / LPR; }
  static __device__ __forceinline__ int col() { return thread() % LPR * 8; }
  static __device__ __forceinline__ bool in(int p) { return RPP <= CHUNK || row(p) < CHUNK; }   // (all threads take part)
  // the first `rows` rows from `base` on, LD elements apart; zeros behind them
  __device__ __forceinline__ void fetch(const T* base, int rows, int ld = D) {
    const unsigned lane = unsigned((thread() / LPR) * ld + col());
    if (RPP <= CHUNK && rows >= CHUNK) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) raw[p].load(base + p * RPP * ld + lane);
      return;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      raw[p].zero();
      if (in(p) && row(p) < rows) raw[p].load(base + p * RPP * ld + lane);
    }
  }
  __device__ __forceinline__ void commit(uint16_t* tile) const {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      bf16x8 x[PARTS];
      raw[p].parts(x);
      if (in(p)) Tile::store8(tile, row(p), col(), x);
    }
  }
  // out[row] = 1 / max(|row|, eps)
  __device__ __forceinline__ void store_factors(float* out, float inv_eps) const {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const float f = row_factor(group_sum<LPR>(raw[p].sum_sq()), inv_eps);
      if (in(p) && thread() % LPR == 0) out[row(p)] = f;
    }
  }
};

// Decays as logarithms to base 2, in 64 bits: 64 of them are added up and differences of those sums taken, and a token that
// forgets everything must not cost the ones behind it their accuracy.  What is below fp32's least number counts as 2^-256.
__device__ __forceinline__ double log2_decay(float log_decay) {
  return log_decay > 0.f ? 0.0 : log_decay < -128.f ? -256.0 : 1.4426950408889634 * double(log_decay);
}
__device__ __forceinline__ float decay_between(double later, double earlier) {
  return __builtin_amdgcn_exp2f(float(later - earlier));
}
// What a state is multiplied by: x times + x plus, with a factor just below 1 as 1 - d and d's own fp32 accuracy.
__device__ __forceinline__ void state_factor(double l2, float& times, float& plus) {
  const float d = -expm1f(float(0.6931471805599453 * l2));
  times = d < 0.5f ? 1.f : __builtin_amdgcn_exp2f(float(l2));
  plus = d < 0.5f ? -d : 0.f;
}

// What a chunk's gates and keys come to, as it lies in the workspace and in LDS.  A decay from row j to a later row i is
// in_tile[i] between[it][jt] to_tile[j] for rows of different tiles of 16, so that tiles below the diagonal take no exponentials
// of their own; none of the three is above 1.
struct alignas(16) ChunkRecord {
  double decay[CHUNK];    // logarithm to base 2 of the decay from the chunk's start to a row, its own included
  float rk[CHUNK];        // 1 / |k|
  float rk_to_tile[CHUNK];   // times the decay behind the row to the end of its tile
  float rk_to_end[CHUNK];    // ... to the end of the chunk
  float rk_since[CHUNK];     // times `since`
  float since[CHUNK];     // the decay from the chunk's start
  float in_tile[CHUNK];   // ... from the start of the row's tile
  float beta[CHUNK];      // 0 where there is no row
  float between[4][4];    // from the end of tile [second] to the start of tile [first]
  float times, plus, unused[2];   // state_factor of the whole chunk
};
constexpr int RECORD_PIECES = sizeof(ChunkRecord) / 16;
static_assert(sizeof(ChunkRecord) == DELTA_RECORD_BYTES && RECORD_PIECES <= 256, "a piece to a thread");

// W as operand fragments of three parts, [fragment][part][lane][8 elements]: of the row (column) tiles 0 .. 3 and the 32 columns
// (rows) ks the ones that are not all zeros.
constexpr int W_FRAGS = 6, W_ELEMS = W_FRAGS * 3 * 64 * 8;
static_assert(2 * W_ELEMS == DELTA_W_BYTES, "workspace");
__host__ __device__ constexpr bool w_row_there(int tile, int ks) { return 2 * ks <= tile; }
__host__ __device__ constexpr int w_row_frag(int tile, int ks) { return (tile < 2 ? tile : 2 * tile - 2) + ks; }
__host__ __device__ constexpr bool w_col_there(int tile, int ks) { return 2 * ks + 1 >= tile; }
__host__ __device__ constexpr int w_col_frag(int tile, int ks) { return tile < 2 ? 2 * tile + ks : tile + 2; }

// The scans' state: a wave holds 16 value columns of it in DK / 16 tiles, keys down, [2 ks + h] with the keys key_of(ks, h, q, v)
// in element v of lane row q: next to each other two tiles are an operand whose slots are 32 consecutive keys, eight to a lane row.
__device__ __forceinline__ constexpr int key_of(int ks, int h, int q, int v) { return 32 * ks + 8 * q + 4 * h + v; }

// A barrier of all waves of a workgroup that orders their LDS accesses, for code that the waves do not share.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// Fragment `at` of an array of fragments of N parts, [fragment][part][lane].
template <int N>
__device__ __forceinline__ void load_frag(const uint16_t* from, int at, int l, bf16x8 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = __builtin_bit_cast(bf16x8, reinterpret_cast<const u32x4*>(from)[(at * N + i) * 64 + l]);
}
template <int N, int M>
__device__ __forceinline__ void store_frag(uint16_t* to, int at, int l, const bf16x8 (&f)[M]) {
#pragma unroll
  for (int i = 0; i < N; ++i) reinterpret_cast<u32x4*>(to)[(at * N + i) * 64 + l] = __builtin_bit_cast(u32x4, f[i]);
}
// A row length as a number that the compiler takes for another one in every step of a loop: the addresses of the step's rows are
// then scalars and one lane offset, not a pair of vector registers to each row all through the loop.
__device__ __forceinline__ int in_this_step(int n) {
  asm volatile("" : "+s"(n));
  return n;
}
__device__ __forceinline__ f32x4 four(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// Chunks of a unit in the workspace.
__host__ __device__ constexpr int delta_chunks(int N) { return (N + CHUNK - 1) / CHUNK; }

}  // namespace
}  // namespace cottn
