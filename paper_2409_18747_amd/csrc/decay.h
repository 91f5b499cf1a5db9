// What the kernels of attention with a decay for each head share.  With g = exp(log_decay[h]) the state
// before row i + 1 is H_i = g H_(i-1) + kh_i^T v_i, so that row j reaches row i with the weight g^(i-j).
//
// A chunk takes rows b .. e-1 (n = e - b of them); H is the state after row b-1 and R = sum over i >= e of
// g^(i-e) qh_i^T dO_i the reverse-time state.  Then with i', j' counted from b
//     o_i   = s [ g^(i'+1) qh_i H + sum_{j<=i} g^(i-j) (qh_i . kh_j) v_j ],   H <- g^n H + sum_j g^(n-1-j') kh_j^T v_j
//     dqh_i = s [ g^(i'+1) dO_i H^T + sum_{j<=i} g^(i-j) (dO_i . v_j) kh_j ]
//     dkh_j = s [ g^(n-j') v_j R^T + sum_{i>=j} g^(i-j) (dO_i . v_j) qh_i ]
//     dv_j  = s [ g^(n-j') kh_j R + sum_{i>=j} g^(i-j) (qh_i . kh_j) dO_i ],  R <- g^n R + sum_i g^i' qh_i^T dO_i
// Every exponent that is formed is one of these, or a part of one that is not negative itself: a weight may
// underflow, none overflows, however strong the decay.
//
// Included behind tile_io.h, and as often.

namespace cottn {
namespace COTTN_NS {

#ifdef COTTN_ELEM_F16
constexpr bool ELEM_IS_F16 = true;
#else
constexpr bool ELEM_IS_F16 = false;
#endif

// The decay of a head as logarithms.  Values above 0 count as 0; one of -inf (nothing is kept) becomes a finite
// number, so that 0 rows later the weight is 1 and not NaN.
struct Decay {
  float ln, l2;
  __device__ __forceinline__ explicit Decay(float log_decay) {
    ln = log_decay > 0.f ? 0.f : log_decay;
    ln = ln < -1e30f ? -1e30f : ln;   // (NaN stays)
    l2 = 1.44269504f * ln;
  }
  // g^n for n >= 0
  __device__ __forceinline__ float after(float n) const { return __builtin_amdgcn_exp2f(l2 * n); }
};

// What a state is multiplied by n rows later: x * times + x * plus.  A factor just below 1 is 1 - d with a d of its own, whose
// relative error is that of fp32: as one rounded number, g^64 of a head that hardly forgets would be off by up to 2^-25 with
// the same sign in every chunk, 3e-5 of what is oldest after 1024 chunks.  x * plus is formed of a finite number in place of an
// infinite x, which then stays x: inf - inf d would be NaN.
__device__ __forceinline__ float made_finite(float x) {
  return __builtin_amdgcn_fmed3f(x, -3.402823466e38f, 3.402823466e38f);   // (of NaN some number: the other term is NaN)
}
struct Kept {
  float times, plus;
  __device__ __forceinline__ Kept(const Decay& g, float n) {
    const float d = -expm1f(g.ln * n);
    const float t = d < 0.5f ? 1.f : g.after(n), p = d < 0.5f ? -d : 0.f;
    times = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, t)));
    plus = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, p)));
  }
  __device__ __forceinline__ f32x4 of(f32x4 x) const {
    f32x4 y;
#pragma unroll
    for (int v = 0; v < 4; ++v) y[v] = __builtin_fmaf(made_finite(x[v]), plus, x[v] * times);
    return y;
  }
  template <int A, int B>
  __device__ __forceinline__ void on(f32x4 (&t)[A][B]) const {
    if (times == 1.f) {   // the same for all lanes
#pragma unroll
      for (int x = 0; x < A; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y)
#pragma unroll
          for (int v = 0; v < 4; ++v) t[x][y][v] = __builtin_fmaf(t[x][y][v], plus, t[x][y][v]);
    } else {
#pragma unroll
      for (int x = 0; x < A; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y)
#pragma unroll
          for (int v = 0; v < 4; ++v) t[x][y][v] *= times;
    }
  }
  // the same, where some element is `infinite` (any_infinite): made_finite for every state of 64 x 16 heads of 2048 rows 128 x
  // 128 took 562 us instead of 547, and 96 units of 1024 rows forward + backward 162 instead of 155
  template <int A, int B>
  __device__ __forceinline__ void on(f32x4 (&t)[A][B], bool infinite) const {
    if (infinite) {
#pragma unroll
      for (int x = 0; x < A; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y) t[x][y] = of(t[x][y]);
    } else {
      on(t);
    }
  }
};
// Whether a wave's part of a state has an infinite element, the same for all lanes.  Only one that a caller hands over is
// looked at: finite rows make none below fp32's largest number.
template <int A, int B>
__device__ __forceinline__ bool any_infinite(const f32x4 (&t)[A][B]) {
  float most = 0.f;
#pragma unroll
  for (int x = 0; x < A; ++x)
#pragma unroll
    for (int y = 0; y < B; ++y)
#pragma unroll
      for (int v = 0; v < 4; ++v) most = fmaxf(most, fabsf(t[x][y][v]));
  return __any(most > 3.402823466e38f);
}

// Rows are raw in LDS and every factor of a row (1 / norm, decay) goes to fp32 results, to the masked tiles before they are
// rounded, or to operand fragments below: an element of a result has met one rounding to 16 bits but for its own.  A product of
// two rows takes their factors one after the other: the two, each up to 1 / eps, may leave fp32 when the product is small, or
// 0.
//   fp16: rows of q and k times the power of two that brings their norm to 16 .. 32 (exact but for elements 2^-18 below the
// norm), so that the factors left, 1/32 .. 1/16, are alike for short and long rows.  The tiles of dO . v take them TILE_UNIT
// times larger, 1/2 .. 1, so that what is rounded is never above the product, nor less than half of it: they leave fp16 for no
// row norm, neither for the 1 / eps of a short row nor for the small ones of a long one, and for no product that fp16 holds.
constexpr float TILE_UNIT = ELEM_IS_F16 ? 16.f : 1.f;
template <class Stage>
struct RowFactors {
  float left[Stage::PASSES];    // what the row in the tile is to be multiplied by
  float whole[Stage::PASSES];   // min(1 / norm, 1 / eps)
  __device__ __forceinline__ void commit(const Stage& stage, lds_t* tile, float inv_eps, Unparted& un) {
    stage.row_rinv(inv_eps, whole);
    if constexpr (ELEM_IS_F16) {
      float power[Stage::PASSES];
#pragma unroll
      for (int p = 0; p < Stage::PASSES; ++p) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, whole[p]);
        power[p] = 32.f * __builtin_bit_cast(float, bits & 0x7F800000u);
        left[p] = 1.f / 32.f * __builtin_bit_cast(float, (bits & 0x007FFFFFu) | 0x3F800000u);
      }
      stage.commit_scaled(tile, power, un);
    } else {
#pragma unroll
      for (int p = 0; p < Stage::PASSES; ++p) left[p] = whole[p];
      stage.commit_plain(tile, un);
    }
  }
};

// An operand fragment whose k slots are tokens, each token's values times a weight, in parts: each the rest that rounding the
// ones before left over.  A state that is a result in fp32, and those that ds is formed from, take EXACT_PARTS, until fp32 has
// no more: three in bfloat16 (two leave up to 2^-17 of a product, 2.4e-6 of a state in the mean), two in fp16, whole fp32 one.
// One that only enters rounded results takes two at most: with one the 1.4 roundings of a result would be 1.7.
#if defined(COTTN_ELEM_F32)
constexpr int EXACT_PARTS = 1, ROUNDED_PARTS = 1;
#elif defined(COTTN_ELEM_F16)
constexpr int EXACT_PARTS = 2, ROUNDED_PARTS = 2;
#else
constexpr int EXACT_PARTS = 3, ROUNDED_PARTS = 2;
#endif
template <int PARTS>
struct WeightedFrag { frag8 part[PARTS]; };
template <int PARTS>
__device__ __forceinline__ WeightedFrag<PARTS> weighted(const frag8& x, const float (&w)[8]) {
  WeightedFrag<PARTS> f;
#if defined(COTTN_F32_WHOLE)
#pragma unroll
  for (int j = 0; j < 8; ++j) f.part[0][j] = x[j] * w[j];
#elif !defined(COTTN_ELEM_F32)
  const u32x4 words = __builtin_bit_cast(u32x4, x);
  u32x4 parts[PARTS];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b, pa, pb;
    unpack2(words[i], a, b);
    parts[0][i] = pack2(a * w[2 * i], b * w[2 * i + 1]);
    unpack2(parts[0][i], pa, pb);
    a = __builtin_fmaf(a, w[2 * i], -pa);
    b = __builtin_fmaf(b, w[2 * i + 1], -pb);
    parts[1][i] = pack2(a, b);
    if constexpr (PARTS > 2) {
      unpack2(parts[1][i], pa, pb);
      parts[2][i] = pack2(a - pa, b - pb);
    }
  }
#pragma unroll
  for (int i = 0; i < PARTS; ++i) f.part[i] = __builtin_bit_cast(frag8, parts[i]);
#endif
  return f;
}
// the weights of the tokens t0 .. t0+3 and t1 .. t1+3
__device__ __forceinline__ void token_weights(const float* of, int t0, int t1, float (&w)[8]) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(of + t0), hi = *reinterpret_cast<const f32x4*>(of + t1);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    w[v] = lo[v];
    w[4 + v] = hi[v];
  }
}

// Accumulators hold states in units of 1 / STATE_UNIT, and the weights that tokens enter them with are as many times larger: in
// fp16 the second part of kh_j g^n, 2^-11 of it, would else lie below the smallest normal number (2^-14) and lose up to 2^-25,
// whatever the weight.  (|kh| <= 1: no product is over 2^14.)
constexpr float STATE_UNIT = ELEM_IS_F16 ? 16384.f : 1.f, PER_UNIT = 1.f / STATE_UNIT;

// The weighted fragments of a wave's key tiles (columns of a tile of k or q rows), for all tokens of a chunk.
template <class ST, int NP, int PITCH, int PARTS>
struct WeightedTile {
  WeightedFrag<PARTS> f[NP][ST::NCT];
  __device__ __forceinline__ WeightedTile(const lds_t* tile, const float* weights, int w, int r, int q4) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
      float wt[8];
      token_weights(weights, t0, t1, wt);
#pragma unroll
      for (int x = 0; x < ST::NCT; ++x) f[p][x] = weighted<PARTS>(lds_col_frag(tile, PITCH, t0, t1, 16 * ST::col_tile(w, x), r), wt);
    }
  }
  // sums(x, y) += (the weighted columns)^T (the value columns of `rows`) for N of the wave's value tiles from y0 on: part by
  // part, the smallest first, so that neighbouring matrix instructions do not wait for each other's sums
  template <int N, int PITCH_V, class Sum>
  __device__ __forceinline__ void add(const lds_t* rows, int y0, int w, int r, int q4, Sum sum) const {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int t0 = 32 * p + 4 * q4, t1 = t0 + 16;
      frag8 v[N];
#pragma unroll
      for (int y = 0; y < N; ++y) v[y] = lds_col_frag(rows, PITCH_V, t0, t1, 16 * ST::row_tile(w, y0 + y), r);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
        for (int x = 0; x < ST::NCT; ++x)
#pragma unroll
          for (int y = 0; y < N; ++y) sum(x, y) = mma16_add(v[y], f[p][x].part[i], sum(x, y));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Fills half of an operand fragment with four values.
__device__ __forceinline__ void put_four(frag8& frag, int half, f32x4 x) {
#if defined(COTTN_F32_WHOLE)
#pragma unroll
  for (int v = 0; v < 4; ++v) frag[4 * half + v] = x[v];
#elif !defined(COTTN_ELEM_F32)
  u32x4 words = __builtin_bit_cast(u32x4, frag);
  words[2 * half + 0] = pack2(x[0], x[1]);
  words[2 * half + 1] = pack2(x[2], x[3]);
  frag = __builtin_bit_cast(frag8, words);
#endif
}

// The states that other workgroups left at the start of segment g: sum over the slots first .. last of g^(seg_rows * (distance
// from `last` or `first`)), nearest slot with weight 1, two at a time with all loads before the first addition.
template <bool REVERSE, int NCT, int NRT, class LoadTile>
__device__ __forceinline__ void add_decayed_states(f32x4 (&acc)[NCT][NRT], int first, int last, const Decay& g, int seg_rows,
                                                   LoadTile load) {
  constexpr int BATCH = states_at_once(NCT * NRT);
  for (int base = first; base <= last; base += BATCH) {
    f32x4 t[BATCH][NCT][NRT];
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
#pragma unroll
      for (int x = 0; x < NCT; ++x)
#pragma unroll
        for (int y = 0; y < NRT; ++y) t[i][x][y] = load(min(base + i, last), x, y);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (base + i > last) break;
      const float w = g.after(float(REVERSE ? base + i - first : last - base - i) * float(seg_rows));
#pragma unroll
      for (int x = 0; x < NCT; ++x)
#pragma unroll
        for (int y = 0; y < NRT; ++y)
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[x][y][v] = __builtin_fmaf(w, t[i][x][y][v], acc[x][y][v]);
    }
  }
}

// A tree of up to 64 drafted tokens, lane l with node l: parent[i] is a node before i; any other value makes i a root.
// path: the node and its ancestors as bits (in the order of their depths, since parents come first).
struct TreeNode {
  unsigned long long path = 0;
  __device__ __forceinline__ TreeNode(const int* __restrict__ parent, int n_tokens, int l) {
    int up = l < n_tokens ? parent[l] : -1;
    up = up >= 0 && up < l ? up : -1;
    path = 1ull << l;
#pragma unroll
    for (int i = 0; i < 6; ++i) {   // paths of 2^i nodes, then of twice as many
      const unsigned long long above = __shfl(path, up < 0 ? l : up, 64);
      const int next = __shfl(up, up < 0 ? l : up, 64);
      path |= above;
      up = next;
    }
  }
  __device__ __forceinline__ int depth() const { return __builtin_popcountll(path) - 1; }
};

// Flags of a scan: what the states are (DecayArgs::carried), and rows that nothing will find in a cache again.
enum : int { CARRIED = 1, STREAM_Q = 2, STREAM_KV = 4, STREAM = 8 };

// waves per SIMD that registers are capped for: two workgroups to a compute unit where the LDS holds them
constexpr int decay_waves(int lds_bytes, int waves, int waves_per_group) {
  const int own = waves / 4 < 1 ? 1 : waves / 4, at_once = (160 * 1024) / lds_bytes >= 2 ? 2 : 1;
  const int most = waves_per_group > 1 ? 4 : 2;
  return own * at_once <= most ? own * at_once : own > most ? own : most;
}

}  // namespace COTTN_NS
}  // namespace cottn
