// gfx950 kernels of the attention of drafted tokens over a fixed-rate key-value cache
// (hq_cache_tree_attention): the last tokens of each sequence are a tree, and every one
// of them attends over the tokens before the tree and over its own ancestors.
//
// The queries of a KV head, `group` of each drafted token, are rows of a tile; a workgroup
// takes one tile of one sequence's head and a chunk of its tokens, each wave 32 tokens at a
// time, as the one-token attention does:
//   scores   C[token, row] = K (16 tokens x 128) Q^T (16 rows)
//   values   O^T[dim, row] += V^T (16 dims x 32 tokens) P^T
// with the same numbering of a step's tokens, so that no weight moves between lanes.
//
// Both products run on the matrix cores in fp16, which holds every int8 and E4M3 code exactly, and an
// MXFP4 code with its block's scale relative to the token's largest as a multiple of 2^-24: of blocks
// 2^-24 of the largest and less it loses codes, 2^-25 of the largest at most.  A query row is
// moved to [2^14, 2^15) by a power of two and enters as two fp16 terms, cut off: 11 + 11 bits
// of the row's largest value.  So do a weight times its token's value scale: a row's reference
// (TreeState, kSlack) keeps that product below 2^15 and its row's largest at 2^1 or more, so
// that two terms, 22 bits of a product or 2^-24 of it, whichever is coarser, cut off no more
// than 2^-21 of the largest.  Scores, references and sums are fp32.  (Three bf16 terms hold all
// 24 bits, for half as many products again and twice the instructions of cutting.)
//
// What bounds it: a row and token take 2 x 2 x 2 x 128 operations of the matrix cores, and a
// lane's 16 of them some 8 instructions each for their softmax, two terms included.  8 sequences of
// 8192 tokens, 64 rows, 8 KV heads of 4, int8: 167 us in tiles of 128 rows and the join's 11.  In 40 %
// of the kernel's cycles the matrix units are busy, in 48 % the vector units.  A wave's products wait
// for its softmax and its softmax for its products, so they overlap with another wave's only, of
// which a SIMD has two.  (The codes' bytes take 29 us at a copy's rate, the two terms' products 116
// at that of a large matrix product.  24 uneven trees in MXFP4, groups of 7, in tiles of 32: 66 us,
// matrix units busy in 23 %, vector units in 52.)
#include <hip/hip_runtime.h>

#include <type_traits>

#include "hq_cache_device.h"
#include "hq_lds.h"

#pragma clang fp contract(off)

namespace {

typedef _Float16 v2h_t __attribute__((ext_vector_type(2)));
typedef _Float16 v8h16_t __attribute__((ext_vector_type(8)));

typedef float v16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ v16_t mfma_f16(const uint4& a, const uint32_t* b, v16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h16_t, a),
                                                __builtin_bit_cast(v8h16_t, (v4w_t){b[0], b[1], b[2], b[3]}), c, 0, 0, 0);
}
__device__ __forceinline__ v4_t mfma_f16(const uint32_t* a, const uint32_t* b, v4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h16_t, (v4w_t){a[0], a[1], a[2], a[3]}),
                                                __builtin_bit_cast(v8h16_t, (v4w_t){b[0], b[1], b[2], b[3]}), c, 0, 0, 0);
}

// Two values as the first and second fp16 terms, cut off.  The first's remainder is exact: an
// fp16 half times -1 plus the fp32 value, one instruction.
__device__ __forceinline__ void two_terms(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));
  float a, b;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(a) : "v"(hi), "v"(x));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(b) : "v"(hi), "v"(y));
  lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

// Int8 codes c + 128 as bytes 0 and 2 of a word, which are the fp16 numbers (c + 128) 2^-24:
// c 2^-9.  The scales take the 2^9 (kCodeUnit), of which one of 2^119 or more becomes infinite; with
// two references (below) a row's scores and its values' sum take it.
__device__ __forceinline__ uint32_t halves_of_bytes(uint32_t w) {
  const v2h_t x = __builtin_bit_cast(v2h_t, w);
  const v2h_t up = {(_Float16)32768.0f, (_Float16)32768.0f}, off = {(_Float16)-0.25f, (_Float16)-0.25f};
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, up, off));
}
template <int FMT>
constexpr float kCodeUnit = FMT == kInt8 ? 512.0f : 1.0f;

// One word's codes as fp16 pairs along the dims: int8 and E4M3 two, MXFP4 four (times `f`).
template <int FMT>
__device__ __forceinline__ void dims_of(uint32_t w, float f, uint32_t* o) {
  if constexpr (FMT == kInt8) {
    const uint32_t x = w ^ 0x80808080u;
    o[0] = halves_of_bytes(__builtin_amdgcn_perm(0u, x, 0x0C010C00u));
    o[1] = halves_of_bytes(__builtin_amdgcn_perm(0u, x, 0x0C030C02u));
  } else if constexpr (FMT == kE4M3) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, f, 0));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, f, 1));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, f, 2));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, f, 3));
  }
}

// Two tokens' words as fp16 pairs (first token, second) per dim: int8 and E4M3 four dims,
// MXFP4 eight (f: the tokens' factors).
template <int FMT>
__device__ __forceinline__ void tokens_of(uint32_t w0, uint32_t w1, float f0, float f1, uint32_t* o) {
  if constexpr (FMT == kInt8) {
    const uint32_t x0 = w0 ^ 0x80808080u, x1 = w1 ^ 0x80808080u;
#pragma unroll
    for (uint32_t d = 0; d < 4; ++d) o[d] = halves_of_bytes(__builtin_amdgcn_perm(x1, x0, 0x0C040C00u + d * 0x00010001u));
  } else {
    constexpr int D = FMT == kMx ? 4 : 2;
    uint32_t a[D], b[D];
    dims_of<FMT>(w0, f0, a);
    dims_of<FMT>(w1, f1, b);
#pragma unroll
    for (int d = 0; d < D; ++d) {
      o[2 * d] = __builtin_amdgcn_perm(b[d], a[d], 0x05040100u);
      o[2 * d + 1] = high_pair(a[d], b[d]);
    }
  }
}

// A step's codes and scales; of MXFP4 a token's scale is its largest block's, and a block's
// factor relative to it.
template <int FMT>
struct TreeStep : CacheStep<FMT> {
  float kf[2], vf[2][4];
};

// The power of two by which 2^(byte - 127) lies below the token's scale (a power of two or NaN).
__device__ __forceinline__ float below_scale(uint32_t byte, float scale) {
  const int32_t e = (int32_t)byte - (int32_t)min(__float_as_uint(scale) >> 23, 255u) + 127;
  return __uint_as_float((uint32_t)max(e, 0) << 23);
}

template <int FMT, bool APART>
__device__ __forceinline__ void tree_take(uint8_t* step, int lane, TreeStep<FMT>& s) {
  using R = CacheRing<FMT>;
  const uint32_t n = lane & 15, g = lane >> 4;
  if constexpr (FMT == kMx) {
    // one lane per token and side: its scale as fp32 into the place of the bytes' first copy.  A
    // wave's LDS operations keep their order, so the fence costs no wait: it holds the compiler
    // from moving the lanes' reads of each other's scales above the writes
    uint8_t* at = step + ((lane >> 4) & 1) * R::HALF + R::SCALES + (lane >> 5) * 256 + n * 4;
    const uint32_t w = *(const uint32_t*)at;
    const uint32_t x = max(max(w & 0xFFu, (w >> 8) & 0xFFu), max((w >> 16) & 0xFFu, w >> 24));
    *(float*)(at + 64) = __uint_as_float(x == 255u ? 0x7FC00000u : x << 23);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  }
  cache_take<FMT>(step, lane, s);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (FMT == kMx) {
      const uint8_t* sc = step + h * R::HALF + R::SCALES + 64;
      const float4 x = *(const float4*)(sc + 16 * g), y = *(const float4*)(sc + 256 + 16 * g);
      s.ks[h][0] = x.x; s.ks[h][1] = x.y; s.ks[h][2] = x.z; s.ks[h][3] = x.w;
      s.vs[h][0] = y.x; s.vs[h][1] = y.y; s.vs[h][2] = y.z; s.vs[h][3] = y.w;
      s.kf[h] = below_scale(s.kx[h], *(const float*)(sc + 4 * n));
#pragma unroll
      for (int r = 0; r < 4; ++r) s.vf[h][r] = below_scale((s.vx[h][r] >> (8 * (n >> 2))) & 0xFFu, s.vs[h][r]);
    } else {
      s.kf[h] = 1.0f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s.vf[h][r] = 1.0f;
        if (!APART) s.ks[h][r] *= kCodeUnit<FMT>;
        if (!APART) s.vs[h][r] *= kCodeUnit<FMT>;
      }
    }
  }
}

// Of two waves of a SIMD the one that is further behind goes first, by quarters of their ways: else
// the older one does throughout, and the younger one's rest runs alone.  (8 sequences of 8192
// tokens and 64 rows: the loops of the first workgroups of the CUs 137 us and of the second 158,
// so 146 and 157; 175.3 us a call to 173.7, 24 uneven trees in MXFP4 72.0 to 70.2.)
struct Behind {
  int32_t left, next, quarter;
  __device__ __forceinline__ void start(int32_t begin, int32_t of) {
    left = 4;
    next = begin;
    quarter = of;
  }
  __device__ __forceinline__ void at(int32_t t, int32_t end) {
    if (t != next) return;
    switch (--left) {
      case 3: __builtin_amdgcn_s_setprio(3); break;
      case 2: __builtin_amdgcn_s_setprio(2); break;
      case 1: __builtin_amdgcn_s_setprio(1); break;
      default: __builtin_amdgcn_s_setprio(0);
    }
    next = left && quarter ? t + quarter : end;
  }
};

// What a row sees, in LDS: only steps that some row does not see some token of look at it.
struct TreeRow {
  uint64_t mask;  // ancestors
  int32_t low;    // first token of its window
  // Bits of the 16 tokens from t on, those before the tree (below ctx) and the tree's.
  __device__ __forceinline__ uint32_t sees(int32_t t, int32_t ctx, int32_t sinks) const {
    auto below = [&](int32_t x) { return (1u << min(max(x - t, 0), 16)) - 1u; };
    const uint32_t before = (below(sinks) | ~below(low)) & below(ctx);
    if (t + 16 <= ctx) return before;
    const int32_t d = t - ctx;  // below 64 where anybody sees a token
    return before | (uint32_t)(d >= 0 ? mask >> (d & 63) : mask << -d);
  }
};

// What a wave carries over its tokens per row tile; acc as in the one-token attention.
struct TreeState {
  float m, l;
  v4_t acc[8];
};

// A row's reference lies above a score by the token's lift, the power of two (as its logarithm)
// that leaves the weight times the value scale below 2^8.  It moves up only when a step's bound
// passes it by 2^7, so that a product stays below 2^15 and the sums are seldom rescaled: with
// 32 rows a wave some row has a new largest score in most steps.  Two terms hold 22 bits of a
// product down to 2^-2, and 2^-24 below.
constexpr float kSlack = 7.0f;

// A scale below 2^-83 stays where it is: products with it are small, and the sum of 2^30 tokens'
// weights of up to 2^97 fits.
__device__ __forceinline__ float lift_of(uint32_t scale_bits) {
  return max((float)((int32_t)((scale_bits >> 23) & 0xFFu) - (126 + 8)), -90.0f);
}

// 2^x of a reference's move, x <= 0, as its root: a sum of weights takes it in two steps.  Zero vectors
// have weights of up to 2^97 under their references, beside a value scale of 2^k others of 2^(7 - k):
// in one step what is left of the first would be 0 from k = 44 on.
__device__ __forceinline__ float half_move(float x) { return __builtin_amdgcn_exp2f(0.5f * x); }

// ---- value scales and scores that one reference does not hold
// It holds value scales from 2^-80 to 2^104: above, weights of 2^-20 of the largest would pass below
// 2^-126, and below, products lose their 22 bits.  And it holds scores (of base 2) up to 2^24, above
// which the lift is lost in a score's rounding.  A wave (of tiles of 128 rows, a workgroup) that met
// a step whose largest scale lies outside, or such a reference, goes over its tokens again with two
// references a row (`apart`): the largest score for the weights, and 2^unit beside it for the
// products, the largest of which lies between 2^7 and 2^8 when it is set.  A product takes an
// exponential of its own there, mantissa(scale) * 2^(score - reference + exponent - unit).  (8
// sequences of 8192 tokens and 64 rows with scales of 2^104: 410 us, 166 with others.)
__device__ __forceinline__ bool scales_apart(uint32_t most) {
  // one comparison for both ends; a zero passes the second
  return most - (47u << 23) > (183u << 23 | 0x7FFFFFu) && most != 0u;
}

__device__ __forceinline__ bool score_apart(float m) { return __builtin_fabsf(m) > 0x1p24f && m != -__builtin_inff(); }

// A value scale's exponent, and its other factor; of a zero vector none.
__device__ __forceinline__ float scale_exp(float s) { return s == 0.0f ? -1000.0f : (float)__builtin_amdgcn_frexp_expf(s); }
__device__ __forceinline__ float scale_mant(float s) { return __builtin_amdgcn_frexp_mantf(s); }

// A row's move: the root of the factor of its sum of weights, and the factor of its values' sum.
struct Move {
  float root, values;
};
// To the largest score `top` and the largest score and exponent `most`(reference) beside it.
template <typename MOST>
__device__ __forceinline__ Move move_apart(float top, float& m, float& unit, MOST most) {
  const float mn = __builtin_fmaxf(m, top), ref = mn == -__builtin_inff() ? 0.0f : mn, by = m - ref;
  const float u = __builtin_fmaxf(__builtin_ceilf(__builtin_fmaxf(unit + by, most(ref) - 8.0f)), -140.0f);
  const Move x = {half_move(by), __builtin_amdgcn_exp2f(by + (unit - u))};
  m = mn;
  unit = u;
  return x;
}

// A weight, which `sum` takes, and its product with a value scale.  x: score - reference, -inf where
// the row does not see the token, whose scale may be a NaN.
__device__ __forceinline__ float product_apart(float x, float scale, float unit, float& sum) {
  sum += __builtin_amdgcn_exp2f(x);
  const float p = scale_mant(scale) * __builtin_amdgcn_exp2f(x + (scale_exp(scale) - unit));
  return x == -__builtin_inff() ? 0.0f : p;
}

// A row's sums with two references as those of one, both within fp32: products of up to 2^8, 2^30
// tokens of them with codes of up to 2^9, have room for 2^80, and what is left goes into the
// reference (which a score above 2^24 rounds away: parts of a row whose value scales lie above 2^87
// then meet with weights that are off by the scales' ratio).  Returns the factor of the values' sum.
__device__ __forceinline__ float join_apart(float unit, float& m, float& l) {
  const float left = __builtin_fminf(__builtin_fmaxf(unit, -80.0f), 80.0f);
  m += unit - left;
  l *= __builtin_amdgcn_exp2f(left - unit);
  return __builtin_amdgcn_exp2f(left);
}

// Whether one lift, the largest scale's, does for tokens whose scales lie between these: the
// largest product of a row is then at least 2^1.
__device__ __forceinline__ bool one_lift(uint32_t least, uint32_t most) { return (least >> 23) + 6 >= most >> 23; }

// 32 tokens' scores in C's layout to their weights' terms pt (k index 4 h + r) and into the
// rows' references and sums.  each: some row does not see some token, or the tokens' value scales
// lie far apart: a lift for each; otherwise `lift` for all.  The sums are rescaled in one place:
// with one for each of two ways the compiler keeps the accumulators twice.
template <int RT>
__device__ __forceinline__ void tree_weights(v4_t (&c)[RT][2], const float (&ks)[2][4], const float (&vs)[2][4], bool each,
                                             float lift, const SpanWalk& w, int32_t t, uint32_t seen, const TreeRow* rows,
                                             const float (&back)[RT], int lane, bool& odd, TreeState (&z)[RT],
                                             uint32_t (&pt)[RT][2][4]) {
  const int g = lane >> 4;
  float top[RT];
  bool more = false;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) c[i][h][r] *= ks[h][r];
  }
  if (each) {
    int32_t live[2], at[2];
    w.about(t, seen, live, at);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const TreeRow row = rows[16 * i + (lane & 15)];
      top[i] = -__builtin_inff();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t sees = (row.sees(at[h], w.ctx, w.sinks) & (uint32_t)live[h]) >> (4 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          c[i][h][r] = (sees >> r) & 1 ? c[i][h][r] : -__builtin_inff();
          top[i] = __builtin_fmaxf(top[i], __builtin_fmaf(c[i][h][r], back[i], lift_of(__float_as_uint(vs[h][r]))));
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      top[i] = c[i][0][0];
#pragma unroll
      for (int k = 1; k < 8; ++k) top[i] = __builtin_fmaxf(top[i], c[i][k >> 2][k & 3]);
      top[i] = __builtin_fmaf(top[i], back[i], lift);
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    top[i] = groups_max(top[i]);
    more |= top[i] > z[i].m + kSlack;
  }
  if (__ballot(more)) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      // a row's own scores alone move it
      const float mn = top[i] > z[i].m + kSlack ? top[i] : z[i].m;
      const float root = half_move(z[i].m - (mn == -__builtin_inff() ? 0.0f : mn)), alpha = root * root;
      z[i].m = mn;
      odd |= __ballot(score_apart(mn)) != 0;
      z[i].l = z[i].l * root * root;
#pragma unroll
      for (int j = 0; j < 8; ++j) z[i].acc[j] *= alpha;
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float ref = z[i].m == -__builtin_inff() ? 0.0f : z[i].m;  // nothing seen yet
    float v[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) v[h][r] = vs[h][r];
    if (each) {
      // a scale that the row does not see may be a NaN
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[h][r] = c[i][h][r] == -__builtin_inff() ? 0.0f : vs[h][r];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(c[i][h][r], back[i], -ref));
        z[i].l += e[r];
      }
#pragma unroll
      for (int r = 0; r < 4; r += 2)
        two_terms(e[r] * v[h][r], e[r + 1] * v[h][r + 1], pt[i][0][2 * h + r / 2], pt[i][1][2 * h + r / 2]);
    }
  }
}

// The same with two references.
template <int RT>
__device__ __forceinline__ void tree_weights_apart(v4_t (&c)[RT][2], const float (&ks)[2][4], const float (&vs)[2][4],
                                                   bool each, const SpanWalk& w, int32_t t, uint32_t seen,
                                                   const TreeRow* rows, const float (&back)[RT], int lane, float (&unit)[RT],
                                                   TreeState (&z)[RT], uint32_t (&pt)[RT][2][4]) {
  const int g = lane >> 4;
  int32_t live[2], at[2];
  w.about(t, seen, live, at);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const TreeRow row = rows[16 * i + (lane & 15)];
    float top = -__builtin_inff();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t sees = each ? (row.sees(at[h], w.ctx, w.sinks) & (uint32_t)live[h]) >> (4 * g) : 15u;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        c[i][h][r] = (sees >> r) & 1 ? c[i][h][r] * ks[h][r] * back[i] : -__builtin_inff();
        top = __builtin_fmaxf(top, c[i][h][r]);
      }
    }
    const Move by = move_apart(groups_max(top), z[i].m, unit[i], [&](float ref) {
      float most = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < 8; ++k) most = __builtin_fmaxf(most, c[i][k >> 2][k & 3] - ref + scale_exp(vs[k >> 2][k & 3]));
      return groups_max(most);
    });
    z[i].l = z[i].l * by.root * by.root;
#pragma unroll
    for (int j = 0; j < 8; ++j) z[i].acc[j] *= by.values;
    const float ref = z[i].m == -__builtin_inff() ? 0.0f : z[i].m;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = product_apart(c[i][h][r] - ref, vs[h][r], unit[i], z[i].l);
#pragma unroll
      for (int r = 0; r < 4; r += 2) two_terms(p[r], p[r + 1], pt[i][0][2 * h + r / 2], pt[i][1][2 * h + r / 2]);
    }
  }
}

// One step: the 32 tokens from t on, of which `seen` is what SpanWalk::fetch returned.  odd: the
// wave has met what one reference does not hold.  unit: of APART.
template <int FMT, int RT, bool APART>
__device__ __forceinline__ void tree_step(TreeStep<FMT>& cur, const SpanWalk& w, int32_t t, uint32_t seen,
                                          const uint32_t (&q)[RT][2][4][4], const TreeRow* rows, const float (&back)[RT],
                                          int lane, bool& odd, float (&unit)[RT], TreeState (&z)[RT]) {
  const int g = lane >> 4;
  bool each = !(seen & 1);  // some row does not see some token
  if (each) {
    int32_t live[2], at[2];
    w.about(t, seen, live, at);
    // tokens that nobody sees: their value codes count as zeros (a stale code may be a NaN)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!((live[h] >> (4 * g + r)) & 1)) {
#pragma unroll
          for (int i = 0; i < CacheStep<FMT>::VW; ++i) cur.v[h][r][i] = 0u;
          cur.ks[h][r] = cur.vs[h][r] = 0.0f;
        }
  }
  float most = cur.vs[0][0], least = most;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    most = __builtin_fmaxf(most, cur.vs[i >> 2][i & 3]);
    least = __builtin_fminf(least, cur.vs[i >> 2][i & 3]);
  }
  const uint32_t hi = readfirst(__float_as_uint(groups_max(most))), lo = readfirst(__float_as_uint(-groups_max(-least)));
  if (!APART) {
    each |= !one_lift(lo, hi);
    odd |= scales_apart(hi);
  }
  v4_t c[RT][2];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) c[i][h] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t a[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (FMT == kMx) {
        dims_of<FMT>(cur.k[h][s], cur.kf[h], a[h]);
      } else {
        dims_of<FMT>(cur.k[h][2 * s], 1.0f, a[h]);
        dims_of<FMT>(cur.k[h][2 * s + 1], 1.0f, a[h] + 2);
      }
    }
#pragma unroll
    for (int t = 1; t >= 0; --t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < RT; ++i) c[i][h] = mfma_f16(a[h], q[i][t][s], c[i][h]);
  }
  uint32_t pt[RT][2][4];
  if constexpr (APART)
    tree_weights_apart<RT>(c, cur.ks, cur.vs, each, w, t, seen, rows, back, lane, unit, z, pt);
  else
    tree_weights<RT>(c, cur.ks, cur.vs, each, lift_of(hi), w, t, seen, rows, back, lane, odd, z, pt);
  // value codes: per word the tokens' pairs of each of its dims
#pragma unroll
  for (int w = 0; w < CacheStep<FMT>::VW; ++w) {
    constexpr int D = 8 / CacheStep<FMT>::VW;  // dims of a word
    uint32_t vf[D][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        uint32_t o[D];
        tokens_of<FMT>(cur.v[h][r][w], cur.v[h][r + 1][w], cur.vf[h][r], cur.vf[h][r + 1], o);
#pragma unroll
        for (int d = 0; d < D; ++d) vf[d][2 * h + r / 2] = o[d];
      }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int t = 1; t >= 0; --t)
#pragma unroll
        for (int d = 0; d < D; ++d) z[i].acc[D * w + d] = mfma_f16(vf[d], pt[i][t], z[i].acc[D * w + d]);
  }
}

// A row of a sequence's tile: its token in the tree and its query head among the KV head's.
struct TreePlace {
  int32_t i, head;  // i: of the tree, at or past its end where the tile has none
  __device__ __forceinline__ TreePlace(const hq_cache_attn_args& A, int32_t row) {
    i = (int32_t)A.by_group.of((uint32_t)row);
    head = row - i * A.group;
  }
};

__device__ __forceinline__ TreeRow tree_row(const hq_cache_attn_args& A, int32_t row, int32_t rows, int32_t from, int32_t ctx) {
  const TreePlace p(A, row);
  uint64_t mask = p.i < rows ? A.masks[from + p.i] : 0;
  if (rows < 64) mask &= (1ull << rows) - 1;
  return {mask, A.window ? ctx + (int32_t)__popcll(mask) - A.window : 0};
}

// 8 values a lane of a query in the cache's coordinates, moved by a power of two so that the
// largest of its 128 lies in [2^14, 2^15), as two terms; returns 1 / that power.
__device__ __forceinline__ float tree_query(const Raw8& raw, bool bf16, uint4 signs, float scale, const TwSigns& sg,
                                            uint4& hi, uint4& lo) {
  float v[8], am = 0.0f;
  expand8(raw, bf16, v);
  flip8(v, signs);
  fwht128_tw(v, sg);
  scale = xor_sign(scale, sg.sigma);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] *= scale;
    am = __builtin_fmaxf(am, __builtin_fabsf(v[k]));
  }
  am = __builtin_fmaxf(am, dpp_xor<1>(am));
  am = __builtin_fmaxf(am, dpp_xor<2>(am));
  am = __builtin_fmaxf(am, swz_xor4(am));
  am = __builtin_fmaxf(am, dpp_xor<8>(am));
  // its exponent, between -100 and 127
  const int32_t e = min(max((int32_t)(__float_as_uint(am) >> 23), 27), 254) - 127;
  const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
  two_terms(v[0] * up, v[1] * up, hi.x, lo.x);
  two_terms(v[2] * up, v[3] * up, hi.y, lo.y);
  two_terms(v[4] * up, v[5] * up, hi.z, lo.z);
  two_terms(v[6] * up, v[7] * up, hi.w, lo.w);
  return __uint_as_float((uint32_t)(127 - 14 + e) << 23);
}

// A row's sum of a chunk, 16 lanes: to the join, or finished.
__device__ __forceinline__ void tree_result(const hq_cache_attn_args& A, bool join, int64_t part, float M, float L, float* v,
                                            const TreePlace& p, int32_t rows, int32_t from, int32_t head, int lane) {
  const int c0 = (lane & 15) * 8;
  if (!join) {
    cache_finish(A, L, v, head, lane);
    if (p.i < rows)
      store8(A.out, ((int64_t)(from + p.i) * A.heads_q + (int64_t)head * A.group + p.head) * HQ_TILE + c0, A.out_bf16, v);
  } else if (p.i < rows) {
    store8(A.part_acc, part * HQ_TILE + c0, false, v);
    if (c0 == 0) {
      A.part_m[part] = M;
      A.part_l[part] = L;
    }
  }
}

template <int FMT, int RT>
constexpr int tree_wave_bytes() {
  constexpr int out = 16 * RT * kOPitch * (int)sizeof(float);
  return CacheRing<FMT>::WAVE > out ? CacheRing<FMT>::WAVE : out;
}

// Tiles of 16 RT rows: every wave has all of them and its own tokens.  (24 uneven trees in MXFP4,
// groups of 7: 69.6 us a call; the longest wave goes through 22 steps, some 5400 cycles each with two
// waves a SIMD.  1 x 777 tokens 11.8 us: four steps and the chain around them.)
template <int FMT, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void hq_cache_tree_kernel(
    hq_cache_attn_args A) {
  using R = CacheRing<FMT>;
  constexpr int ROWS = 16 * RT, WAVE = tree_wave_bytes<FMT, RT>();
  extern __shared__ __attribute__((aligned(16))) uint8_t s_ring[];  // a wave's ring after the other
  __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS], s_f[ROWS];
  __shared__ TreeRow s_row[ROWS];
  // term t of row tile i lies in the second step of wave 2 i + t's ring until that is first
  // loaded, a wave's sums in its own ring at the end
  static_assert(16 * kQPitch * sizeof(uint16_t) <= R::STEP && 2 * RT <= WAVES, "");
  auto q_row = [&](int row, int t) {
    return (uint16_t*)(s_ring + (2 * (row >> 4) + t) * WAVE + R::STEP) + (row & 15) * kQPitch;
  };
  auto o_row = [&](int w, int row) { return (float*)(s_ring + w * WAVE) + row * kOPitch; };
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4, grp = tid >> 4;
  const int wave = (int)readfirst((uint32_t)(tid >> 6));
  const int32_t j = (int32_t)(blockIdx.x / (uint32_t)A.heads_kv), c0 = n * 8;
  const int32_t head = (int32_t)(blockIdx.x - (uint32_t)j * (uint32_t)A.heads_kv);
  const CacheItem it = cache_item<kTree>(A, j, lane, blockIdx.x == 0 && wave == 0);
  if (it.b < 0) return;
  // what the join goes by
  if (A.join && A.batch <= HQ_CACHE_UNPLANNED && j == it.first && head == 0 && tid == 0)
    A.parts[it.b] = {it.first, it.n};
  const int32_t rows = it.span.rows, seen = it.span.seen(), tile = it.tile;
  if (tile * ROWS >= rows * A.group) return;  // none of this sequence's, or it has none at all
  const int32_t from = it.span.from;
  const int32_t begin0 = (int32_t)(it.at * it.chunk), tokens = min(it.chunk, seen - begin0);
  const int32_t per = (tokens + 32 * WAVES - 1) / (32 * WAVES) * 32;
  const int32_t end = begin0 + min(tokens, (wave + 1) * per), begin = min(begin0 + wave * per, end);
  SpanWalk w;
  w.start(A, it, head, begin);
  w.ask(A, begin, lane);
  Raw8 qraw[RT] = {};
  const uint4 qd = sign_words(A.k_dsign16, head * HQ_TILE + c0);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const TreePlace p(A, tile * ROWS + 16 * i + grp);
    if (grp < 16 && p.i < rows)
      qraw[i] = load_raw8(A.q, ((int64_t)(from + p.i) * A.heads_q + (int64_t)head * A.group + p.head) * HQ_TILE + c0, A.q_bf16);
  }
  if (tid < ROWS) s_row[tid] = tree_row(A, tile * ROWS + tid, rows, from, w.ctx);
  w.got();
  uint8_t* ring = s_ring + wave * WAVE;
  uint32_t sees = 0, next = 0;
  if (begin < end) sees = w.template fetch<FMT>(A, begin, end, lane, ring);
  // ---- the queries into the cache's coordinates, as two fp16 terms of a power of two times each
  const TwSigns sg(lane);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    if (grp >= 16) break;  // the last four of eight waves
    uint4 hi, lo;
    const float f = tree_query(qraw[i], A.q_bf16, qd, A.qscale, sg, hi, lo);
    *(uint4*)(q_row(16 * i + grp, 0) + c0) = hi;
    *(uint4*)(q_row(16 * i + grp, 1) + c0) = lo;
    if (n == 0) s_f[16 * i + grp] = f;
  }
  __syncthreads();
  // step s of the contraction takes dims 32 (l / 16) + 8 s + j in lane l (the codes
  // that the lane's one run of 32 holds)
  uint32_t q[RT][2][4][4];
  float back[RT];  // 1 / the power of two that a row was moved by
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint4 x = *(const uint4*)(q_row(16 * i + n, t) + 32 * g + 8 * s);
        q[i][t][s][0] = x.x; q[i][t][s][1] = x.y; q[i][t][s][2] = x.z; q[i][t][s][3] = x.w;
      }
    back[i] = s_f[16 * i + n];
  }
  __syncthreads();  // the queries' place is loaded over

  TreeState z[RT];
  bool odd = false;
  float unit[RT] = {};
  auto way = [&](auto apart) {
    constexpr bool APART = decltype(apart)::value;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      z[i].m = -__builtin_inff();
      z[i].l = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i].acc[k] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (begin + 32 < end) next = w.template fetch<FMT>(A, begin + 32, end, lane, ring + R::STEP);
    int32_t slot = 0;
    Behind first;
    first.start(begin, (end - begin) / 128 * 32);
    for (int32_t t = begin; t < end; t += 32) {
      first.at(t, end);
      // the loads of this step are done when at most the next step's are not
      if (t + 32 < end)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R::LOADS) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      TreeStep<FMT> cur;
      tree_take<FMT, APART>(ring + slot * R::STEP, lane, cur);
      const uint32_t here = sees;
      sees = next;
      if (t + 64 < end) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what the ring held is in registers
        next = w.template fetch<FMT>(A, t + 64, end, lane, ring + slot * R::STEP);
      }
      slot ^= 1;
      tree_step<FMT, RT, APART>(cur, w, t, here, q, s_row, back, lane, odd, unit, z);
    }
  };
  way(std::false_type());
  if (__builtin_expect(odd, 0)) {
#pragma unroll
    for (int i = 0; i < RT; ++i) back[i] *= kCodeUnit<FMT>;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what the ring held is in registers
    w.ask(A, begin, lane);
    w.got();
    sees = w.template fetch<FMT>(A, begin, end, lane, ring);
    way(std::true_type());
  }
  // ---- the waves' sums under one reference, one row per 16 lanes
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    z[i].l = groups_sum(z[i].l);
    if (odd) {
      const float by = kCodeUnit<FMT> * join_apart(unit[i], z[i].m, z[i].l);
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i].acc[k] *= by;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* o = o_row(wave, 16 * i + n) + (4 * g + r) * 8;
      *(float4*)o = make_float4(z[i].acc[0][r], z[i].acc[1][r], z[i].acc[2][r], z[i].acc[3][r]);
      *(float4*)(o + 4) = make_float4(z[i].acc[4][r], z[i].acc[5][r], z[i].acc[6][r], z[i].acc[7][r]);
    }
    if (g == 0) {
      s_m[wave][16 * i + n] = z[i].m;
      s_l[wave][16 * i + n] = z[i].l;
    }
  }
  __syncthreads();
  if (grp >= 16) return;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int at_row = 16 * i + grp;
    const TreePlace p(A, tile * ROWS + at_row);
    float M = s_m[0][at_row], L = 0.0f, v[8] = {};
#pragma unroll
    for (int x = 1; x < WAVES; ++x) M = __builtin_fmaxf(M, s_m[x][at_row]);
    const float ref = M == -__builtin_inff() ? 0.0f : M;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      const float root = half_move(s_m[x][at_row] - ref), f = root * root;
      L = __builtin_fmaf(root, root * s_l[x][at_row], L);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(f, o_row(x, at_row)[c0 + k], v[k]);
    }
    tree_result(A, it.n > 1, (int64_t)blockIdx.x * ROWS + at_row, M, L, v, p, rows, from, head, lane);
  }
}

// ---- many rows
// Tiles of 128 rows of a KV head, 32 of each wave: the codes are turned into fp16 once per
// workgroup and not once per wave.  A workgroup goes through its tokens in tiles of 64, two
// steps of 32; each wave turns the keys and values of 16 of them into LDS in the order that the
// products' operands are read in, a tile ahead of the products; the codes of the tile after it
// are on their way in registers meanwhile.  (8 sequences of 8192 tokens and 64 rows, groups of 4:
// 172 us a call, and 181 in tiles of 32 rows, whose waves each turn what they read.  Tiles of 256 rows,
// eight waves of one workgroup a CU, were 3 % faster there, but took 299 for uneven trees where these
// took 221.)
//
// The products are 32 x 32 x 16: a step's scores are one tile C[token, row], in which lane l
// holds tokens 8 q + 4 (l / 32) + r of row l % 32; with product t of the values contracting
// tokens 16 t .. in the order 8 q' + 4 (l / 32) + r, lane by lane, they are its operand's.
constexpr int kTreeTile = 64, kWideRows = 128;
template <int FMT>
struct TreeTile {
  // keys: [step][contraction step][lane] 16 bytes, dims 8 (2 s + l / 32) ..;  values: [step][group
  // of 32 dims][product][lane] 16 bytes, group d being dims 8 (l % 16) + 2 d + l / 16 % 2
  static constexpr int V = kTreeTile * HQ_TILE * 2, KS = 2 * V, VS = KS + 4 * kTreeTile, SEEN = VS + 4 * kTreeTile;
  static constexpr int BYTES = SEEN + 4 * 16 + 448;  // a multiple of 1 KB
};

// A wave's 16 tokens of a tile on their way: lane l has 32 codes of key l % 16 (run l / 16) and 8
// dims (8 (l % 16) ..) of the four values 8 (l / 32) + 4 (l / 16 % 2) + r.
template <int FMT>
struct TreeLoads {
  static constexpr int KW = FMT == kMx ? 4 : 8, VW = FMT == kMx ? 1 : 2;
  uint32_t k[KW], v[4][VW];
  uint32_t ks, vs;  // scales of token l % 16
  int32_t live;     // bits of tokens that anybody sees
};

// A wave's way over its tokens of a workgroup's tiles.
struct TreeWay {
  const int32_t* table;
  CacheSpan span;
  int32_t gap, jump, head, last;  // last: the sequence's last block
  int32_t id;                     // the next tile's block, on its way
  __device__ __forceinline__ int32_t real(int32_t t) const { return t < jump ? t : t + gap; }
  __device__ __forceinline__ void ask(const hq_cache_attn_args& A, int32_t t) {
    id = table[min((int32_t)A.by_block.of((uint32_t)real(t)), last)];
  }
  // Starts the loads of the 16 tokens from t on, whose block has been asked for, and asks for
  // that of the tile behind.
  template <int FMT>
  __device__ __forceinline__ void load(const hq_cache_attn_args& A, int32_t t, int32_t end, int lane, TreeLoads<FMT>& x) {
    constexpr int RB = row_bytes<FMT>();
    const int n = lane & 15, g = lane >> 4;
    const int32_t at = real(t), blk = (int32_t)readfirst((uint32_t)id);
    const bool in = t < end, bad = (uint32_t)blk >= (uint32_t)A.blocks;
    if (in && bad && head == 0 && lane == 0) report(A.stats, HQ_ERR_INVALID_ARG);
    x.live = in && !bad ? (int32_t)span.bits(at) : 0;
    // 16 tokens that nobody sees: the cache's first ones
    const int32_t off = at - (int32_t)A.by_block.of((uint32_t)at) * A.block_tokens;
    const int64_t row = x.live ? ((int64_t)blk * A.heads_kv + head) * A.block_tokens + off : 0;
    ask(A, t + kTreeTile);
    const uint8_t *k = uniform(A.k_codes, row * RB), *v = uniform(A.v_codes, row * RB);
    const uint32_t lk = n * RB + g * (RB / 4), lv = (8 * (g >> 1) + 4 * (g & 1)) * RB + n * (RB / 16);
#pragma unroll
    for (int i = 0; i < TreeLoads<FMT>::KW; i += 4) {
      const uint4 w = *(const uint4*)(k + (lk + 4 * i));
      x.k[i] = w.x; x.k[i + 1] = w.y; x.k[i + 2] = w.z; x.k[i + 3] = w.w;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (FMT == kMx) {
        x.v[r][0] = *(const uint32_t*)(v + (lv + r * RB));
      } else {
        const uint2 w = *(const uint2*)(v + (lv + r * RB));
        x.v[r][0] = w.x; x.v[r][1] = w.y;
      }
    }
    x.ks = *(const uint32_t*)(uniform(A.k_scales, row * 4) + 4 * (uint32_t)n);
    x.vs = *(const uint32_t*)(uniform(A.v_scales, row * 4) + 4 * (uint32_t)n);
  }
};

__device__ __forceinline__ uint32_t largest_byte(uint32_t w) {
  return max(max(w & 0xFFu, (w >> 8) & 0xFFu), max((w >> 16) & 0xFFu, w >> 24));
}
// Bits of a token's scale: MXFP4's is its largest block's.
template <int FMT, bool APART>
__device__ __forceinline__ uint32_t token_scale(uint32_t w) {
  if constexpr (FMT == kMx) {
    const uint32_t x = largest_byte(w);
    return x == 255u ? 0x7FC00000u : x << 23;
  } else {
    return APART ? w : __float_as_uint(__uint_as_float(w) * kCodeUnit<FMT>);
  }
}

// The largest of 16 neighbouring lanes' values.
__device__ __forceinline__ float row_max(float x) {
  x = __builtin_fmaxf(x, dpp_xor<1>(x));
  x = __builtin_fmaxf(x, dpp_xor<2>(x));
  x = __builtin_fmaxf(x, swz_xor4(x));
  return __builtin_fmaxf(x, dpp_xor<8>(x));
}

// The 16 tokens as fp16 into a tile, where they are its `group`-th, with their scales and what
// the products go by: the value scales' largest and least, and the tokens that anybody sees.
template <int FMT, bool APART>
__device__ __forceinline__ void turn(TreeLoads<FMT>& x, uint8_t* tile, int group, int lane) {
  using T = TreeTile<FMT>;
  constexpr int VW = TreeLoads<FMT>::VW, D = 8 / VW;
  const int n = lane & 15, g = lane >> 4, step = group >> 1, h = group & 1;
  const uint32_t ks = token_scale<FMT, APART>(x.ks);
  uint32_t vs = token_scale<FMT, APART>(x.vs);
  const float kf = FMT == kMx ? below_scale((x.ks >> (8 * g)) & 0xFFu, __uint_as_float(ks)) : 1.0f;
  float vf[4] = {1.0f, 1.0f, 1.0f, 1.0f};
  if constexpr (FMT == kMx) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int from = 8 * (g >> 1) + 4 * (g & 1) + r;  // a lane that has the token's
      const uint32_t w = (uint32_t)__shfl((int)x.vs, from, 64), of = (uint32_t)__shfl((int)vs, from, 64);
      vf[r] = below_scale((w >> (8 * (n >> 2))) & 0xFFu, __uint_as_float(of));
    }
  }
  if (x.live != 0xFFFF) {
    // tokens that nobody sees count as zeros (a stale code or scale may be a NaN)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!((x.live >> (8 * (g >> 1) + 4 * (g & 1) + r)) & 1)) {
#pragma unroll
        for (int i = 0; i < VW; ++i) x.v[r][i] = 0u;
      }
    if (!((x.live >> n) & 1)) vs = 0u;
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t o[4];
    if constexpr (FMT == kMx) {
      dims_of<FMT>(x.k[s], kf, o);
    } else {
      dims_of<FMT>(x.k[2 * s], 1.0f, o);
      dims_of<FMT>(x.k[2 * s + 1], 1.0f, o + 2);
    }
    // dims 8 (4 g + s) ..
    *(uint4*)(tile + ((step * 8 + 2 * g + s / 2) * 64 + (s & 1) * 32 + 16 * h + n) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
  }
#pragma unroll
  for (int w = 0; w < VW; ++w) {
    uint32_t o[2][D];
#pragma unroll
    for (int r = 0; r < 2; ++r) tokens_of<FMT>(x.v[2 * r][w], x.v[2 * r + 1][w], vf[2 * r], vf[2 * r + 1], o[r]);
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int j = D * w + d;  // dim 8 n + j
      *(uint2*)(tile + T::V + (((step * 4 + j / 2) * 2 + h) * 64 + (g & 1) * 32 + (j & 1) * 16 + n) * 16 + (g >> 1) * 8) =
          make_uint2(o[0][d], o[1][d]);
    }
  }
  if (g == 0) {
    *(uint32_t*)(tile + T::KS + (group * 16 + n) * 4) = ks;
    *(uint32_t*)(tile + T::VS + (group * 16 + n) * 4) = vs;
  }
  const float most = row_max(__uint_as_float(vs)), least = -row_max(-__uint_as_float(vs));
  if (lane == 0)
    *(uint4*)(tile + T::SEEN + group * 16) = make_uint4(__float_as_uint(most), __float_as_uint(least), (uint32_t)x.live, 0u);
}

// Everything that the workgroup wrote to LDS is there for all of it; loads from memory stay on their way.
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a wave carries over its tokens: a lane's row's reference and sum, its values' sum, acc[d][i]
// dim 8 (8 (i / 4 % 2) + 4 (l / 32) + i % 4) + 2 d + i / 8.
struct WideState {
  float m, l;
  v16_t acc[4];
};

// tree_weights of 32 tokens' scores in the 32 x 32 layout; ks and vs in LDS; pt: the terms of the
// two products' operands.
__device__ __forceinline__ void wide_weights(v16_t& c, const float* ks, const float* vs, bool each, float lift,
                                             const int32_t (&live)[2], const int32_t (&at)[2], int32_t ctx, int32_t sinks,
                                             const TreeRow* rows, float back, int lane, uint32_t& odd, WideState& z,
                                             uint32_t (&pt)[2][2][4]) {
  const int u = lane >> 5;
  float top;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 k = *(const float4*)(ks + 8 * q + 4 * u);
    c[4 * q] *= k.x; c[4 * q + 1] *= k.y; c[4 * q + 2] *= k.z; c[4 * q + 3] *= k.w;
  }
  if (each) {
    const TreeRow row = rows[lane & 31];
    top = -__builtin_inff();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t sees = (row.sees(at[h], ctx, sinks) & (uint32_t)live[h]) >> (4 * u);
#pragma unroll
      for (int q = 2 * h; q < 2 * h + 2; ++q) {
        const float4 v = *(const float4*)(vs + 8 * q + 4 * u);
        const float v4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          c[4 * q + r] = (sees >> (8 * (q & 1) + r)) & 1 ? c[4 * q + r] : -__builtin_inff();
          top = __builtin_fmaxf(top, __builtin_fmaf(c[4 * q + r], back, lift_of(__float_as_uint(v4[r]))));
        }
      }
    }
  } else {
    top = c[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = __builtin_fmaxf(top, c[k]);
    top = __builtin_fmaf(top, back, lift);
  }
  const v2u_t t = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
  top = __builtin_fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
  if (__ballot(top > z.m + kSlack)) {
    // a row's own scores alone move it
    const float mn = top > z.m + kSlack ? top : z.m;
    const float root = half_move(z.m - (mn == -__builtin_inff() ? 0.0f : mn)), alpha = root * root;
    z.m = mn;
    if (score_apart(mn)) odd = 1u;
    z.l = z.l * root * root;
#pragma unroll
    for (int d = 0; d < 4; ++d) z.acc[d] *= alpha;
  }
  const float ref = z.m == -__builtin_inff() ? 0.0f : z.m;  // nothing seen yet
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 v = *(const float4*)(vs + 8 * q + 4 * u);
    float w[4] = {v.x, v.y, v.z, v.w};
    if (each) {
      // a scale that the row does not see may be a NaN
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = c[4 * q + r] == -__builtin_inff() ? 0.0f : w[r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(c[4 * q + r], back, -ref));
      z.l += e;
      w[r] *= e;
    }
    two_terms(w[0], w[1], pt[0][q / 2][2 * (q & 1)], pt[1][q / 2][2 * (q & 1)]);
    two_terms(w[2], w[3], pt[0][q / 2][2 * (q & 1) + 1], pt[1][q / 2][2 * (q & 1) + 1]);
  }
}

// The same with two references.
__device__ __forceinline__ void wide_weights_apart(v16_t& c, const float* ks, const float* vs, bool each,
                                                   const int32_t (&live)[2], const int32_t (&at)[2], int32_t ctx,
                                                   int32_t sinks, const TreeRow* rows, float back, int lane, float& unit,
                                                   WideState& z, uint32_t (&pt)[2][2][4]) {
  const int u = lane >> 5;
  auto both = [](float x) {
    const v2u_t t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
  };
  const TreeRow row = rows[lane & 31];
  float top = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int h = k >> 3, token = 8 * (k >> 2) + 4 * u + (k & 3);
    const uint32_t sees = each ? row.sees(at[h], ctx, sinks) & (uint32_t)live[h] : 0xFFFFu;
    c[k] = (sees >> (token & 15)) & 1 ? c[k] * ks[token] * back : -__builtin_inff();
    top = __builtin_fmaxf(top, c[k]);
  }
  const Move by = move_apart(both(top), z.m, unit, [&](float ref) {
    float most = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < 16; ++k) most = __builtin_fmaxf(most, c[k] - ref + scale_exp(vs[8 * (k >> 2) + 4 * u + (k & 3)]));
    return both(most);
  });
  z.l = z.l * by.root * by.root;
#pragma unroll
  for (int d = 0; d < 4; ++d) z.acc[d] *= by.values;
  const float ref = z.m == -__builtin_inff() ? 0.0f : z.m;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = product_apart(c[4 * q + r] - ref, vs[8 * q + 4 * u + r], unit, z.l);
    two_terms(p[0], p[1], pt[0][q / 2][2 * (q & 1)], pt[1][q / 2][2 * (q & 1)]);
    two_terms(p[2], p[3], pt[0][q / 2][2 * (q & 1) + 1], pt[1][q / 2][2 * (q & 1) + 1]);
  }
}

// What a workgroup keeps in LDS beside its tiles.
struct WideShared {
  float m[kWideRows], l[kWideRows], f[kWideRows];
  TreeRow row[kWideRows];
  uint32_t odd;  // some wave has met what one reference does not hold
};
typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef __attribute__((address_space(3))) WideShared lds_wide;
typedef __attribute__((address_space(4))) const hq_cache_attn_args kernel_args;

// Workgroup `block` of the grid.  Returns whether it has to be done over again with two references.
template <int FMT, bool APART>
__device__ __forceinline__ bool wide_workgroup(const hq_cache_attn_args& A, uint32_t block, int tid, uint8_t* s_tile,
                                               WideShared& S) {
  using T = TreeTile<FMT>;
  constexpr int ROWS = kWideRows;
  static_assert(ROWS * kOPitch * (int)sizeof(float) <= 2 * T::BYTES && ROWS * 2 * HQ_TILE * 2 <= 2 * T::BYTES, "");
  auto o_row = [&](int row) { return (float*)s_tile + row * kOPitch; };
  const int lane = tid & 63, n = lane & 15, grp = tid >> 4;
  const int wave = (int)readfirst((uint32_t)(tid >> 6));
  const int32_t j = (int32_t)(block / (uint32_t)A.heads_kv), c0 = n * 8;
  const int32_t head = (int32_t)(block - (uint32_t)j * (uint32_t)A.heads_kv);
  const CacheItem it = cache_item<kTree>(A, j, lane, block == 0 && wave == 0);
  if (it.b < 0) return false;
  // what the join goes by
  if (A.join && A.batch <= HQ_CACHE_UNPLANNED && j == it.first && head == 0 && tid == 0)
    A.parts[it.b] = {it.first, it.n};
  const int32_t rows = it.span.rows, seen = it.span.seen(), tile = it.tile;
  if (tile * ROWS >= rows * A.group) return false;  // none of this sequence's, or it has none at all
  const int32_t from = it.span.from;
  const int32_t begin = (int32_t)(it.at * it.chunk), end = begin + min(it.chunk, seen - begin);
  TreeWay way;
  way.table = A.table + (int64_t)it.b * A.max_blocks;
  way.span = it.span;
  way.gap = it.span.gap();
  way.jump = way.gap ? it.span.turn() : 0x7FFFFFFF;
  way.head = head;
  way.last = (it.span.len - 1) / A.block_tokens;
  TreeLoads<FMT> loads;
  way.ask(A, begin + 16 * wave);
  way.template load<FMT>(A, begin + 16 * wave, end, lane, loads);
  const int32_t ctx = it.span.len - rows;
  if (tid < ROWS) S.row[tid] = tree_row(A, tile * ROWS + tid, rows, from, ctx);
  if (tid == 0) S.odd = 0u;
  // ---- the queries into the cache's coordinates, as two fp16 terms of a power of two times each,
  // [32 rows][term][contraction step][lane] 16 bytes; the next ones are on their way meanwhile
  const uint4 qd = sign_words(A.k_dsign16, head * HQ_TILE + c0);
  auto query = [&](int i) {
    const TreePlace p(A, tile * ROWS + 16 * i + grp);
    Raw8 raw = {};
    if (i < ROWS / 16 && p.i < rows)
      raw = load_raw8(A.q, ((int64_t)(from + p.i) * A.heads_q + (int64_t)head * A.group + p.head) * HQ_TILE + c0, A.q_bf16);
    return raw;
  };
  Raw8 raw0 = query(0), raw1 = query(1);
  const TwSigns sg(lane);
#pragma unroll 1
  for (int i = 0; i < ROWS / 16; ++i) {
    const Raw8 raw = raw0;
    raw0 = raw1;
    raw1 = query(i + 2);
    uint4 hi, lo;
    const float f = tree_query(raw, A.q_bf16, qd, A.qscale, sg, hi, lo);
    uint8_t* to = s_tile + (i >> 1) * 16384 + (n >> 1) * 1024 + ((n & 1) * 32 + (i & 1) * 16 + grp) * 16;
    *(uint4*)to = hi;
    *(uint4*)(to + 8192) = lo;
    if (n == 0) S.f[16 * i + grp] = f;
  }
  __syncthreads();
  uint32_t q[2][8][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const uint4 x = *(const uint4*)(s_tile + ((wave * 2 + t) * 8 + s) * 1024 + lane * 16);
      q[t][s][0] = x.x; q[t][s][1] = x.y; q[t][s][2] = x.z; q[t][s][3] = x.w;
    }
  // 1 / the power of two that the row was moved by
  const float back = S.f[32 * wave + (lane & 31)] * (APART ? kCodeUnit<FMT> : 1.0f);
  __syncthreads();  // the queries' place is written over
  WideState z;
  // from here on every row's window has begun
  const int32_t open = A.window ? ctx + rows - A.window : 0;
  const bool idle = tile * ROWS + 32 * wave >= rows * A.group;  // the wave has no rows
  float unit = 0.0f;
  z.m = -__builtin_inff();
  z.l = 0.0f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int k = 0; k < 16; ++k) z.acc[d][k] = 0.0f;
  turn<FMT, APART>(loads, s_tile, wave, lane);
  if (begin + kTreeTile < end) way.template load<FMT>(A, begin + kTreeTile + 16 * wave, end, lane, loads);
  tile_barrier();
  uint8_t* at_tile = s_tile;
  uint8_t* to_tile = s_tile + T::BYTES;
  Behind first;
  first.start(begin, (end - begin) / (4 * kTreeTile) * kTreeTile);
  for (int32_t t = begin; t < end; t += kTreeTile) {
    first.at(t, end);
    if (t + kTreeTile < end) {
      turn<FMT, APART>(loads, to_tile, wave, lane);
      if (t + 2 * kTreeTile < end) way.template load<FMT>(A, t + 2 * kTreeTile + 16 * wave, end, lane, loads);
    }
#pragma unroll 1
    for (int step = 0; step < 2; ++step) {
      const uint4 about0 = *(const uint4*)(at_tile + T::SEEN + step * 32);
      const uint4 about1 = *(const uint4*)(at_tile + T::SEEN + step * 32 + 16);
      const int32_t live[2] = {(int32_t)readfirst(about0.z), (int32_t)readfirst(about1.z)};
      if ((live[0] | live[1]) == 0 || idle) continue;
      // the largest and least value scale: not negative, so ordered as their bits are
      const uint32_t most = max(readfirst(about0.x), readfirst(about1.x));
      const uint32_t least = min(readfirst(about0.y), readfirst(about1.y));
      const int32_t at[2] = {way.real(t + 32 * step), way.real(t + 32 * step + 16)};
      bool each = (live[0] & live[1]) != 0xFFFF || (!APART && !one_lift(least, most));
#pragma unroll
      for (int h = 0; h < 2; ++h) each |= at[h] + 16 > ctx || (at[h] < open && at[h] + 16 > A.sinks);
      if (!APART && __builtin_expect(scales_apart(most), 0)) S.odd = 1u;
      v16_t c;
#pragma unroll
      for (int k = 0; k < 16; ++k) c[k] = 0.0f;
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const uint4 a = *(const uint4*)(at_tile + ((step * 8 + s) * 64 + lane) * 16);
#pragma unroll
        for (int t1 = 1; t1 >= 0; --t1) c = mfma_f16(a, q[t1][s], c);
      }
      uint32_t pt[2][2][4];
      const float *ks = (const float*)(at_tile + T::KS) + step * 32, *vs = (const float*)(at_tile + T::VS) + step * 32;
      if constexpr (APART)
        wide_weights_apart(c, ks, vs, each, live, at, ctx, A.sinks, S.row + 32 * wave, back, lane, unit, z, pt);
      else
        wide_weights(c, ks, vs, each, lift_of(most), live, at, ctx, A.sinks, S.row + 32 * wave, back, lane, S.odd, z, pt);
      // the next fragments are read before a product waits for its own
      uint4 v[3];
      auto read = [&](int i) {
        v[i % 3] = *(const uint4*)(at_tile + T::V + (((step * 4 + (i & 3)) * 2 + (i >> 2)) * 64 + lane) * 16);
      };
#pragma unroll
      for (int i = 0; i < 3; ++i) read(i);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int t1 = 1; t1 >= 0; --t1) z.acc[i & 3] = mfma_f16(v[i % 3], pt[t1][i >> 2], z.acc[i & 3]);
        if (i + 3 < 8) read(i + 3);
      }
    }
    tile_barrier();
    uint8_t* const x = at_tile;
    at_tile = to_tile;
    to_tile = x;
  }
  const bool odd = !APART && readfirst(S.odd) != 0u;
  // ---- the sums, one row per 16 lanes
  {
    const v2u_t l = __builtin_amdgcn_permlane32_swap(__float_as_uint(z.l), __float_as_uint(z.l), false, false);
    const int u = lane >> 5, at_row = 32 * wave + (lane & 31);
    float sum = __uint_as_float(l[0]) + __uint_as_float(l[1]);
    if constexpr (APART) {
      const float by = kCodeUnit<FMT> * join_apart(unit, z.m, sum);
#pragma unroll
      for (int d = 0; d < 4; ++d) z.acc[d] *= by;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // i / 4 % 2 = k / 4, i % 4 = k % 4
      const int i = 4 * (k >> 2) + (k & 3);
      float* o = o_row(at_row) + (8 * (k >> 2) + 4 * u + (k & 3)) * 8;
      *(float4*)o = make_float4(z.acc[0][i], z.acc[0][i + 8], z.acc[1][i], z.acc[1][i + 8]);
      *(float4*)(o + 4) = make_float4(z.acc[2][i], z.acc[2][i + 8], z.acc[3][i], z.acc[3][i + 8]);
    }
    if (u == 0) {
      S.m[at_row] = z.m;
      S.l[at_row] = sum;
    }
  }
  __syncthreads();
#pragma unroll 2
  for (int i = 0; i < ROWS / 16; ++i) {
    const int at_row = 16 * i + grp;
    const TreePlace p(A, tile * ROWS + at_row);
    float v[8];
    load8(o_row(at_row), c0, false, v);
    tree_result(A, it.n > 1, (int64_t)block * ROWS + at_row, S.m[at_row], S.l[at_row], v, p, rows, from, head, lane);
  }
  return odd;
}

// A function of its own: as part of the kernel it would cost its loop registers, 2 to 4 % of every call's
// time.  The registers that it saves are the kernel's scratch memory, which other calls do not touch:
// 476 bytes a lane, of which the runtime sets 240 MB aside for a hardware queue.
template <int FMT>
__device__ __attribute__((noinline)) void wide_again(kernel_args* A, uint32_t block, int tid, lds_byte* tile, lds_wide* S) {
  const uint64_t at = (uint64_t)A;  // what is the same in every lane, told so
  const auto* args = (kernel_args*)((uint64_t)readfirst((uint32_t)(at >> 32)) << 32 | readfirst((uint32_t)at));
  auto* t = (lds_byte*)(uintptr_t)readfirst((uint32_t)(uintptr_t)tile);
  auto* s = (lds_wide*)(uintptr_t)readfirst((uint32_t)(uintptr_t)S);
  wide_workgroup<FMT, true>(*(const hq_cache_attn_args*)args, readfirst(block), tid, (uint8_t*)t, *(WideShared*)s);
}

template <int FMT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void hq_cache_tree_wide_kernel(hq_cache_attn_args A) {
  extern __shared__ __attribute__((aligned(16))) uint8_t s_tile[];  // two tiles
  __shared__ WideShared S;
  if (__builtin_expect((wide_workgroup<FMT, false>(A, blockIdx.x, threadIdx.x, s_tile, S)), 0)) {
    __syncthreads();  // the sums have been read
    wide_again<FMT>((kernel_args*)__builtin_amdgcn_kernarg_segment_ptr(), blockIdx.x, threadIdx.x, (lds_byte*)s_tile,
                    (lds_wide*)&S);
  }
}

// Joins the chunks of a row under one reference, in order, and moves the result back: a wave
// per row of a split sequence, 16 lanes for every fourth chunk, whose first four are loaded
// together.  (16 chunks of 32 rows: 11.6 us with 16 lanes for all of a row's chunks.)
__global__ __launch_bounds__(256) void hq_cache_tree_join_kernel(hq_cache_attn_args A, uint32_t per) {
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4, c0 = n * 8;
  int64_t b = blockIdx.x / per;
  const uint32_t at = readfirst((blockIdx.x - (uint32_t)b * per) * 4 + (tid >> 6));  // query head of a drafted token
  if (A.batch > HQ_CACHE_UNPLANNED) {
    if (b >= A.split[A.joins]) return;
    b = A.split[b];
  }
  const hq_cache_of has = A.parts[b];
  if (has.n == 1) return;  // already whole
  const int32_t from = A.starts[b], rows = A.starts[b + 1] - from;
  if (at >= (uint32_t)rows * (uint32_t)A.heads_q) return;
  const uint32_t i = at / (uint32_t)A.heads_q, hq = at - i * (uint32_t)A.heads_q, head = A.by_group.of(hq);
  const uint32_t row = i * (uint32_t)A.group + hq - head * (uint32_t)A.group, tile = row >> A.tile_shift;
  const int64_t part0 = ((((int64_t)has.first + tile) * A.heads_kv + head) << A.tile_shift) + (row - (tile << A.tile_shift));
  const int64_t step = (int64_t)cache_tiles<kTree>(A, rows) * A.heads_kv << A.tile_shift;
  float M = -__builtin_inff(), m[4], l[4], a[4][8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int32_t x = g + 4 * k;
    m[k] = M;
    l[k] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[k][e] = 0.0f;
    if (x >= has.n) continue;
    const int64_t part = part0 + x * step;
    m[k] = A.part_m[part];
    l[k] = A.part_l[part];
    load8(A.part_acc, part * HQ_TILE + c0, false, a[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) M = __builtin_fmaxf(M, m[k]);
  for (int32_t x = g + 16; x < has.n; x += 4) M = __builtin_fmaxf(M, A.part_m[part0 + x * step]);
  M = groups_max(M);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
  float L = 0.0f, v[8] = {};
  auto add = [&](float mx, float lx, const float* ax) {
    const float root = half_move(mx - ref), f = root * root;
    L = __builtin_fmaf(root, root * lx, L);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(f, ax[e], v[e]);
  };
#pragma unroll
  for (int k = 0; k < 4; ++k) add(m[k], l[k], a[k]);
  for (int32_t x = g + 16; x < has.n; x += 4) {
    const int64_t part = part0 + x * step;
    float ax[8];
    load8(A.part_acc, part * HQ_TILE + c0, false, ax);
    add(A.part_m[part], A.part_l[part], ax);
  }
  L = groups_sum(L);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = groups_sum(v[e]);
  cache_finish(A, L, v, (int32_t)head, lane);
  if (g == 0) store8(A.out, ((int64_t)(from + (int32_t)i) * A.heads_q + hq) * HQ_TILE + c0, A.out_bf16, v);
}

template <int FMT, int RT, int WAVES>
int launch_narrow(const hq_cache_attn_args& a, hipStream_t st) {
  static hq_lds_granted granted;
  constexpr size_t lds = (size_t)WAVES * tree_wave_bytes<FMT, RT>();
  if (const int e = hq_allow_lds((const void*)hq_cache_tree_kernel<FMT, RT, WAVES>, lds, granted)) return e;
  hipLaunchKernelGGL((hq_cache_tree_kernel<FMT, RT, WAVES>), dim3((uint32_t)(a.items * a.heads_kv)), dim3(64 * WAVES), lds, st, a);
  return 0;
}

template <int FMT>
int launch_wide(const hq_cache_attn_args& a, hipStream_t st) {
  static hq_lds_granted granted;
  constexpr size_t lds = 2 * TreeTile<FMT>::BYTES;
  if (const int e = hq_allow_lds((const void*)hq_cache_tree_wide_kernel<FMT>, lds, granted)) return e;
  hipLaunchKernelGGL((hq_cache_tree_wide_kernel<FMT>), dim3((uint32_t)(a.items * a.heads_kv)), dim3(256), lds, st, a);
  return 0;
}

template <int FMT>
int launch_tree(const hq_cache_attn_args& a, hipStream_t st) {
  switch (a.tile_shift) {
    case 4:
      // as the one-token attention, calls that leave CUs idle have eight waves share a chunk
      return a.items * a.heads_kv <= 256 ? launch_narrow<FMT, 1, 2 * HQ_CACHE_WAVES>(a, st)
                                         : launch_narrow<FMT, 1, HQ_CACHE_WAVES>(a, st);
    case 5: return launch_narrow<FMT, 2, HQ_CACHE_WAVES>(a, st);
    default: return launch_wide<FMT>(a, st);
  }
}

}  // namespace

int hq_launch_cache_tree(const hq_cache_attn_args& a, int format, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  int e = 0;
  if (a.join && a.batch > HQ_CACHE_UNPLANNED) hq_launch_cache_plan(a, stream);
  switch (format) {
    case HQ_INT8: e = launch_tree<kInt8>(a, st); break;
    case HQ_E4M3: e = launch_tree<kE4M3>(a, st); break;
    default: e = launch_tree<kMx>(a, st);
  }
  if (e) return e;
  if (a.join && a.joins) {
    const uint32_t per = ((uint32_t)a.max_rows * (uint32_t)a.heads_q + 3) / 4;
    hipLaunchKernelGGL(hq_cache_tree_join_kernel, dim3((uint32_t)a.joins * per), dim3(256), 0, st, a, per);
  }
  return (int)hipGetLastError();
}
