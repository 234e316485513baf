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
// Both products run on the matrix cores in fp16, which holds every code of the three formats
// exactly (MXFP4's with its block's scale relative to the token's largest).  A query row is
// moved to [2^14, 2^15) by a power of two and enters as two fp16 terms, cut off: 11 + 11 bits
// of the row's largest value.  So do the weights: a row's reference is the largest score plus
// the power of two of the token's value scale, so that a weight times that scale lies below
// 2^15, and what two terms cut off, 2^-21 of it, is below 2^-21 of the largest term that the
// row sums.  Scores, references and sums are fp32.  (Three bf16 terms hold all 24 bits, for
// half as many products again and twice the instructions of cutting.)
#include <hip/hip_runtime.h>

#include "hq_cache_device.h"
#include "hq_lds.h"

#pragma clang fp contract(off)

namespace {

typedef _Float16 v2h_t __attribute__((ext_vector_type(2)));
typedef _Float16 v8h16_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v4_t mfma_f16(const uint32_t* a, const uint32_t* b, v4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h16_t, (v4w_t){a[0], a[1], a[2], a[3]}),
                                                __builtin_bit_cast(v8h16_t, (v4w_t){b[0], b[1], b[2], b[3]}), c, 0, 0, 0);
}

// Two values as the first and second fp16 terms, cut off; the first's remainder is exact.
__device__ __forceinline__ void two_terms(float x, float y, uint32_t& hi, uint32_t& lo) {
  const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
  const auto l = __builtin_amdgcn_cvt_pkrtz(x - (float)h[0], y - (float)h[1]);
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, l);
}

// Int8 codes c + 128 as bytes 0 and 2 of a word, which are the fp16 numbers (c + 128) 2^-24:
// c 2^-9.  The scales take the 2^9 (kCodeUnit).
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
  float lift[2][4];  // the power of two that moves a token's value scale below 2^15
};

// The power of two by which 2^(byte - 127) lies below the token's scale (a power of two or NaN).
__device__ __forceinline__ float below_scale(uint32_t byte, float scale) {
  const int32_t e = (int32_t)byte - (int32_t)min(__float_as_uint(scale) >> 23, 255u) + 127;
  return __uint_as_float((uint32_t)max(e, 0) << 23);
}

template <int FMT>
__device__ __forceinline__ void tree_take(uint8_t* step, int lane, TreeStep<FMT>& s) {
  using R = CacheRing<FMT>;
  const uint32_t n = lane & 15, g = lane >> 4;
  if constexpr (FMT == kMx) {
    // one lane per token and side: its scale as fp32 into the place of the bytes' first copy
    uint8_t* at = step + ((lane >> 4) & 1) * R::HALF + R::SCALES + (lane >> 5) * 256 + n * 4;
    const uint32_t w = *(const uint32_t*)at;
    const uint32_t x = max(max(w & 0xFFu, (w >> 8) & 0xFFu), max((w >> 16) & 0xFFu, w >> 24));
    *(uint32_t*)(at + 64) = x == 255u ? 0x7FC00000u : x << 23;
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
        s.ks[h][r] *= kCodeUnit<FMT>;
        s.vs[h][r] *= kCodeUnit<FMT>;
      }
    }
  }
}

// What a lane knows of its column's row in each row tile.
struct TreeRow {
  uint64_t mask;  // ancestors
  int32_t low;    // first token of its window
  float f;        // 1 / the power of two that its query was moved by
};

// What a wave carries over its tokens per row tile; acc as in the one-token attention.
struct TreeState {
  float m, l;
  v4_t acc[8];
};

// One step: 32 tokens.  `each`: some row does not see some token.
template <int FMT, int RT>
__device__ __forceinline__ void tree_step(TreeStep<FMT>& cur, const int32_t (&live)[2], const int32_t (&at)[2], bool each,
                                          int32_t ctx, int32_t sinks, const uint32_t (&q)[RT][2][4][4],
                                          const TreeRow (&row)[RT], int lane, TreeState (&z)[RT]) {
  const int g = lane >> 4;
  if (each) {
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
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      // a scale below 2^-80 stays where it is: weights times it are small, sums of the weights alone fit
      cur.lift[h][r] = max((float)((int32_t)((__float_as_uint(cur.vs[h][r]) >> 23) & 0xFFu) - (126 + 15)), -94.0f);
  v4_t c[RT][2];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) c[i][h] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t a[4];
      if constexpr (FMT == kMx) {
        dims_of<FMT>(cur.k[h][s], cur.kf[h], a);
      } else {
        dims_of<FMT>(cur.k[h][2 * s], 1.0f, a);
        dims_of<FMT>(cur.k[h][2 * s + 1], 1.0f, a + 2);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 1; t >= 0; --t) c[i][h] = mfma_f16(a, q[i][t][s], c[i][h]);
    }
  uint32_t pt[RT][2][4];  // the weights' terms: k index 4 h + r
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    TreeState& y = z[i];
    bool gone[2][4];
    float x[2][4], top = -__builtin_inff();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[h][r] = c[i][h][r] * cur.ks[h][r];
        float u = __builtin_fmaf(x[h][r], row[i].f, cur.lift[h][r]);
        if (each) {
          const int32_t t = at[h] + 4 * g + r, d = t - ctx;
          const bool sees = d < 0 ? t >= row[i].low || t < sinks : (bool)((row[i].mask >> (d & 63)) & 1);
          gone[h][r] = !sees || !((live[h] >> (4 * g + r)) & 1);
          u = gone[h][r] ? -__builtin_inff() : u;
        }
        top = __builtin_fmaxf(top, u);
      }
    top = groups_max(top);
    if (__ballot(top > y.m)) {
      const float mn = __builtin_fmaxf(y.m, top);
      const float alpha = __builtin_amdgcn_exp2f(y.m - (mn == -__builtin_inff() ? 0.0f : mn));
      y.m = mn;
      y.l *= alpha;
#pragma unroll
      for (int j = 0; j < 8; ++j) y.acc[j] *= alpha;
    }
    const float ref = y.m == -__builtin_inff() ? 0.0f : y.m;  // nothing seen yet
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h][r], row[i].f, -ref));
        w[r] = e * cur.vs[h][r];
        if (each) {
          e = gone[h][r] ? 0.0f : e;
          w[r] = gone[h][r] ? 0.0f : w[r];
        }
        y.l += e;
      }
#pragma unroll
      for (int r = 0; r < 4; r += 2) two_terms(w[r], w[r + 1], pt[i][0][2 * h + r / 2], pt[i][1][2 * h + r / 2]);
    }
  }
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
    i = row / A.group;
    head = row - i * A.group;
  }
};

template <int FMT, int RT>
constexpr int tree_wave_bytes() {
  constexpr int out = 16 * RT * kOPitch * (int)sizeof(float);
  return CacheRing<FMT>::WAVE > out ? CacheRing<FMT>::WAVE : out;
}

template <int FMT, int RT>
__global__ __launch_bounds__(64 * HQ_CACHE_WAVES) __attribute__((amdgpu_waves_per_eu(2))) void hq_cache_tree_kernel(
    hq_cache_attn_args A) {
  using R = CacheRing<FMT>;
  constexpr int WAVES = HQ_CACHE_WAVES, ROWS = 16 * RT, WAVE = tree_wave_bytes<FMT, RT>();
  extern __shared__ __attribute__((aligned(16))) uint8_t s_ring[];  // a wave's ring after the other
  __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS], s_f[ROWS];
  // term t of row tile i lies in the second step of wave 2 i + t's ring until that is first
  // loaded, a wave's sums in its own ring at the end
  static_assert(16 * kQPitch * sizeof(uint16_t) <= R::STEP && 2 * RT <= WAVES, "");
  auto q_row = [&](int row, int t) {
    return (uint16_t*)(s_ring + (2 * (row >> 4) + t) * WAVE + R::STEP) + (row & 15) * kQPitch;
  };
  auto o_row = [&](int w, int row) { return (float*)(s_ring + w * WAVE) + row * kOPitch; };
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4, grp = tid >> 4;
  const int wave = (int)readfirst((uint32_t)(tid >> 6));
  const int32_t j = (int32_t)(blockIdx.x / (uint32_t)A.units);
  const int32_t unit = (int32_t)(blockIdx.x - (uint32_t)j * (uint32_t)A.units);
  const int32_t tile = unit / A.heads_kv, head = unit - tile * A.heads_kv, c0 = n * 8;
  const CacheItem it = cache_item<kTree>(A, j, lane, blockIdx.x == 0 && wave == 0);
  if (it.b < 0) return;
  // what the join goes by
  if (A.join && A.batch <= HQ_CACHE_UNPLANNED && j == it.first && unit == 0 && tid == 0)
    A.parts[it.b] = {it.first, it.n};
  const int32_t rows = it.span.rows, seen = it.span.seen();
  if (tile * ROWS >= rows * A.group) return;  // none of this sequence's, or it has none at all
  const int32_t from = A.starts[it.b];
  const int32_t begin0 = (int32_t)((j - it.first) * it.chunk), tokens = min(it.chunk, seen - begin0);
  const int32_t per = (tokens + 32 * WAVES - 1) / (32 * WAVES) * 32;
  const int32_t end = begin0 + min(tokens, (wave + 1) * per), begin = min(begin0 + wave * per, end);
  CacheWalk<kTree> w;
  w.table = A.table + (int64_t)it.b * A.max_blocks;
  w.head = head;
  w.start(A, it.span, begin);
  w.ask(lane);
  Raw8 qraw[RT] = {};
  const uint4 qd = sign_words(A.k_dsign16, head * HQ_TILE + c0);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const TreePlace p(A, tile * ROWS + 16 * i + grp);
    if (p.i < rows)
      qraw[i] = load_raw8(A.q, ((int64_t)(from + p.i) * A.heads_q + (int64_t)head * A.group + p.head) * HQ_TILE + c0, A.q_bf16);
  }
  const int32_t ctx = it.span.len - rows;
  TreeRow row[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const TreePlace p(A, tile * ROWS + 16 * i + n);
    const uint64_t mask = p.i < rows ? A.masks[from + p.i] : 0;
    row[i].mask = rows < 64 ? mask & ((1ull << rows) - 1) : mask;
    row[i].low = A.window ? ctx + __popcll(row[i].mask) - A.window : 0;
  }
  w.got();
  w.template enter<FMT, true>(A, lane);
  uint8_t* ring = s_ring + wave * WAVE;
  int32_t live[2], at[2], next[2] = {0, 0}, next_at[2] = {0, 0};
  if (begin < end) w.template fetch<FMT>(A, begin, end, lane, ring, live, at);
  // ---- the queries into the cache's coordinates, as two fp16 terms of a power of two times each
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    float qv[8];
    expand8(qraw[i], A.q_bf16, qv);
    flip8(qv, qd);
    const XSigns sg(lane);
    fwht128(qv, sg);
    float am = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      qv[k] *= A.qscale;
      am = __builtin_fmaxf(am, __builtin_fabsf(qv[k]));
    }
    am = __builtin_fmaxf(am, dpp_xor<1>(am));
    am = __builtin_fmaxf(am, dpp_xor<2>(am));
    am = __builtin_fmaxf(am, swz_xor4(am));
    am = __builtin_fmaxf(am, dpp_xor<8>(am));
    // its exponent, between -100 and 127
    const int32_t e = min(max((int32_t)(__float_as_uint(am) >> 23), 27), 254) - 127;
    const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
    uint4 hi, lo;
    two_terms(qv[0] * up, qv[1] * up, hi.x, lo.x);
    two_terms(qv[2] * up, qv[3] * up, hi.y, lo.y);
    two_terms(qv[4] * up, qv[5] * up, hi.z, lo.z);
    two_terms(qv[6] * up, qv[7] * up, hi.w, lo.w);
    *(uint4*)(q_row(16 * i + grp, 0) + c0) = hi;
    *(uint4*)(q_row(16 * i + grp, 1) + c0) = lo;
    if (n == 0) s_f[16 * i + grp] = __uint_as_float((uint32_t)(127 - 14 + e) << 23);
  }
  __syncthreads();
  // step s of the contraction takes dims 32 (l / 16) + 8 s + j in lane l (the codes
  // that the lane's one run of 32 holds)
  uint32_t q[RT][2][4][4];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint4 x = *(const uint4*)(q_row(16 * i + n, t) + 32 * g + 8 * s);
        q[i][t][s][0] = x.x; q[i][t][s][1] = x.y; q[i][t][s][2] = x.z; q[i][t][s][3] = x.w;
      }
    row[i].f = s_f[16 * i + n];
  }
  __syncthreads();  // the queries' place is loaded over

  TreeState z[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    z[i].m = -__builtin_inff();
    z[i].l = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) z[i].acc[k] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
  }
  // from here on every row's window has begun
  const int32_t open = A.window ? ctx + rows - A.window : 0;
  if (begin + 32 < end) w.template fetch<FMT>(A, begin + 32, end, lane, ring + R::STEP, next, next_at);
  int32_t slot = 0;
  for (int32_t t = begin; t < end; t += 32) {
    // the loads of this step are done when at most the next step's are not
    if (t + 32 < end)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R::LOADS) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    TreeStep<FMT> cur;
    tree_take<FMT>(ring + slot * R::STEP, lane, cur);
    const int32_t here[2] = {live[0], live[1]}, here_at[2] = {at[0], at[1]};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      live[h] = next[h];
      at[h] = next_at[h];
    }
    if (t + 64 < end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what the ring held is in registers
      w.template fetch<FMT>(A, t + 64, end, lane, ring + slot * R::STEP, next, next_at);
    }
    slot ^= 1;
    bool each = (here[0] & here[1]) != 0xFFFF;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      each |= here_at[h] + 16 > ctx || (here_at[h] < open && here_at[h] + 16 > A.sinks);
    tree_step<FMT, RT>(cur, here, here_at, each, ctx, A.sinks, q, row, lane, z);
  }
  // ---- the waves' sums under one reference, one row per 16 lanes
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    z[i].l = groups_sum(z[i].l);
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
      const float f = __builtin_amdgcn_exp2f(s_m[x][at_row] - ref);
      L = __builtin_fmaf(f, s_l[x][at_row], L);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(f, o_row(x, at_row)[c0 + k], v[k]);
    }
    if (it.n > 1) {
      if (p.i >= rows) continue;
      const int64_t part = (int64_t)blockIdx.x * ROWS + at_row;
      store8(A.part_acc, part * HQ_TILE + c0, false, v);
      if (n == 0) {
        A.part_m[part] = M;
        A.part_l[part] = L;
      }
      continue;
    }
    cache_finish(A, L, v, head, lane);
    if (p.i < rows)
      store8(A.out, ((int64_t)(from + p.i) * A.heads_q + (int64_t)head * A.group + p.head) * HQ_TILE + c0, A.out_bf16, v);
  }
}

// Joins the chunks of a row under one reference, in order, and moves the result back: 16
// lanes per row of a split sequence.
__global__ __launch_bounds__(256) void hq_cache_tree_join_kernel(hq_cache_attn_args A, int32_t tile_rows, uint32_t per) {
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, c0 = n * 8;
  int64_t b = blockIdx.x / per;
  const uint32_t at = (blockIdx.x - (uint32_t)b * per) * 16 + (tid >> 4);  // query head of a drafted token
  if (A.batch > HQ_CACHE_UNPLANNED) {
    if (b >= A.split[A.joins]) return;
    b = A.split[b];
  }
  const hq_cache_of has = A.parts[b];
  if (has.n == 1) return;  // already whole
  const int32_t from = A.starts[b], rows = A.starts[b + 1] - from;
  const bool in = at < (uint32_t)rows * (uint32_t)A.heads_q;
  const uint32_t q = in ? at : 0u, i = q / (uint32_t)A.heads_q, hq = q - i * (uint32_t)A.heads_q, head = hq / (uint32_t)A.group;
  const uint32_t row = i * (uint32_t)A.group + hq - head * (uint32_t)A.group, tile = row / (uint32_t)tile_rows;
  const int64_t part0 = ((int64_t)has.first * A.units + tile * (uint32_t)A.heads_kv + head) * tile_rows + (row - tile * (uint32_t)tile_rows);
  const int64_t step = (int64_t)A.units * tile_rows;
  float M = -__builtin_inff();
  for (int32_t x = 0; x < has.n; ++x) M = __builtin_fmaxf(M, A.part_m[part0 + x * step]);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
  float L = 0.0f, v[8] = {};
  for (int32_t x = 0; x < has.n; ++x) {
    const int64_t part = part0 + x * step;
    const float f = __builtin_amdgcn_exp2f(A.part_m[part] - ref);
    float a[8];
    load8(A.part_acc, part * HQ_TILE + c0, false, a);
    L = __builtin_fmaf(f, A.part_l[part], L);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(f, a[e], v[e]);
  }
  cache_finish(A, L, v, (int32_t)head, lane);
  if (in) store8(A.out, ((int64_t)(from + (int32_t)i) * A.heads_q + hq) * HQ_TILE + c0, A.out_bf16, v);
}

template <int FMT, int RT>
int launch_tree(const hq_cache_attn_args& a, hipStream_t st) {
  static hq_lds_granted granted;
  constexpr size_t lds = (size_t)HQ_CACHE_WAVES * tree_wave_bytes<FMT, RT>();
  if (const int e = hq_allow_lds((const void*)hq_cache_tree_kernel<FMT, RT>, lds, granted)) return e;
  hipLaunchKernelGGL((hq_cache_tree_kernel<FMT, RT>), dim3((uint32_t)(a.items * a.units)), dim3(64 * HQ_CACHE_WAVES), lds, st, a);
  return 0;
}

template <int FMT>
int launch_tree(const hq_cache_attn_args& a, hipStream_t st) {
  return hq_tree_tile(a.max_rows * a.group) == 16 ? launch_tree<FMT, 1>(a, st) : launch_tree<FMT, 2>(a, st);
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
    const uint32_t per = ((uint32_t)a.max_rows * (uint32_t)a.heads_q + 15) / 16;
    hipLaunchKernelGGL(hq_cache_tree_join_kernel, dim3((uint32_t)a.joins * per), dim3(256), 0, st, a,
                       hq_tree_tile(a.max_rows * a.group), per);
  }
  return (int)hipGetLastError();
}
