// gfx950 kernels of the fixed-rate key-value cache: rows cast into slots
// (hq_cache_write), read back (hq_cache_read), and one query token per sequence
// attending over a paged cache (hq_cache_attention), or over the last tokens and the first
// ones of it (hq_cache_window_attention, the same kernel with other tokens to go through).
//
// A stored head vector is the cast of y = H D x (H the 128-point Sylvester
// matrix, D the plan's signs of the head's columns): int8 or E4M3 codes c with one
// fp32 scale s, y = s c, or MXFP4.  H D / sqrt(128) is orthogonal, so
//   q . x = (H D q) . y / 128     and     sum_t p_t x_t = D H (sum_t p_t y_t) / 128:
// the attention moves each query once and each output back once, and works on
// the codes as they lie.  Rows lie as [block, head, token of the block], so one head's
// tokens of a block are one run of memory.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "hq_cache_device.h"
#include "hq_lds.h"

#pragma clang fp contract(off)

namespace {

// ------------------------------------------------------------- write and read
// 16 lanes take one head vector, 8 values each; a wave four of them, neighbouring
// heads of one token where there are four.

// A lane group takes two vectors, whose slots and rows are loaded together: with one
// a wave waits for a slot and then for what it points to with little else in flight.
// (65536 rows of 8 heads in int8: written in 78 us with two, 85 with one, read in 44 and
// 56; up to 4096 rows the same.  Four write 8192 rows in 15.1 us, two in 13.4.)
// Both kernels are bound by memory and by VALU issue at once, about 350 instructions
// per pair: 8192 rows of 8 heads from bf16 to E4M3 take 13.4 us (3.8 TB/s), 32768 rows of
// int8 to bf16 23.2 us (4.4 TB/s), where a large copy moves 5.2 TB/s.
constexpr int U = 2;
constexpr uint32_t kIoTiles = 16 * U;  // of a workgroup

struct CacheTiles {
  uint32_t row[U], head[U];  // of the call; past its end the last tile's
  bool in[U];                // not past the end
  int64_t slot[U];
  __device__ __forceinline__ explicit CacheTiles(const hq_cache_io_args& A) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t t = (blockIdx.x * U + i) * 16u + (threadIdx.x >> 4), tile = min(t, A.tiles - 1);
      in[i] = t < A.tiles;
      row[i] = A.by_heads.of(tile);
      head[i] = tile - row[i] * (uint32_t)A.heads;
      slot[i] = A.slots[row[i]];
    }
  }
  // Whether tile i has a slot in the cache, and where its vector lies.
  __device__ __forceinline__ bool at(const hq_cache_io_args& A, const hq_cache_side& S, int lane, int i,
                                     int64_t& vec) const {
    const bool ok = slot[i] >= 0 && slot[i] < S.slots;
    if (slot[i] >= S.slots && head[i] == 0 && (lane & 15) == 0) report(S.stats, HQ_ERR_INVALID_ARG);
    const uint32_t s = ok ? (uint32_t)slot[i] : 0u, blk = A.by_block.of(s);
    vec = (int64_t)(blk * (uint64_t)(uint32_t)A.heads + head[i]) * A.block_tokens + (s - blk * (uint32_t)A.block_tokens);
    return ok && in[i];
  }
};

template <int FMT>
__global__ __launch_bounds__(256) void hq_cache_write_kernel(hq_cache_io_args A) {
  const hq_cache_side& S = A.side[blockIdx.y];
  const int lane = threadIdx.x & 63, c0 = (lane & 15) * 8;
  const CacheTiles t(A);
  float v[U][8];
  uint4 d[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    load8(S.x, (int64_t)t.row[i] * S.ld + (t.head[i] * HQ_TILE + c0), A.x_bf16, v[i]);
    d[i] = sign_words(S.dsign16, t.head[i] * HQ_TILE + c0);
  }
  const TwSigns sg(lane);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    // every lane of a wave stays for the transform's lane moves, which leave sigma
    // times the values
    int64_t vec;
    const bool live = t.at(A, S, lane, i, vec);
    flip8(v[i], d[i]);
    fwht128_tw(v[i], sg);
    cache_put<FMT>(S, v[i], live, vec, lane, sg);
  }
}

// 1 / 128 of the factor that an E8M0 byte stands for: 2^(byte - 134), NaN for 255.  Bytes
// below 8 give subnormal factors; a code times one is a multiple of 2^-135 and exact.
__device__ __forceinline__ float e8m0_128th(uint32_t byte) {
  return byte == 255u ? __builtin_nanf("") : __uint_as_float(byte < 8u ? 1u << (byte + 15u) : (byte - 7u) << 23);
}

template <int FMT>
__global__ __launch_bounds__(256) void hq_cache_read_kernel(hq_cache_io_args A) {
  const hq_cache_side& S = A.side[0];
  const int lane = threadIdx.x & 63, c0 = (lane & 15) * 8;
  const CacheTiles t(A);
  uint2 w[U];
  uint4 d[U];
  float scale[U];  // of the transformed codes
  bool live[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    int64_t vec;  // a vector of the cache also where the tile has none
    live[i] = t.at(A, S, lane, i, vec);
    if constexpr (FMT == kMx) {
      w[i].x = *(const uint32_t*)(S.codes + vec * row_bytes<FMT>() + c0 / 2);
      w[i].y = ((const uint8_t*)S.scales)[vec * 4 + ((lane & 15) >> 2)];
    } else {
      w[i] = *(const uint2*)(S.codes + vec * row_bytes<FMT>() + c0);
      scale[i] = ((const float*)S.scales)[vec];
    }
    d[i] = sign_words(S.dsign16, t.head[i] * HQ_TILE + c0);
  }
  const TwSigns sg(lane);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    float v[8];
    if constexpr (FMT == kMx) {
      // the blocks' factors and the 1 / 128 before H: sums of vectors near the largest that
      // can be written (X up to 125) would pass fp32 without it
      const float f = e8m0_128th(w[i].y);
      const v2f_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, 1.0f, 0);
      const v2f_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, 1.0f, 1);
      const v2f_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, 1.0f, 2);
      const v2f_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, 1.0f, 3);
      v[0] = a[0] * f; v[1] = a[1] * f; v[2] = b[0] * f; v[3] = b[1] * f;
      v[4] = c[0] * f; v[5] = c[1] * f; v[6] = d[0] * f; v[7] = d[1] * f;
    } else {
      const uint32_t w2[2] = {w[i].x, w[i].y};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (FMT == kE4M3) {
          const v2f_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w2[h], false);
          const v2f_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w2[h], true);
          v[4 * h] = a[0]; v[4 * h + 1] = a[1]; v[4 * h + 2] = b[0]; v[4 * h + 3] = b[1];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * h + e] = (float)(int8_t)(w2[h] >> (8 * e));
        }
      }
    }
    fwht128_tw(v, sg);
    // int8 and E4M3: H of the codes first, then the scale: integer codes sum exactly
    const float f = xor_sign(FMT == kMx ? 1.0f : scale[i] * 0.0078125f, sg.sigma);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= f;
    flip8(v, d[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = live[i] ? v[e] : 0.0f;
    if (t.in[i]) store8(A.y, (int64_t)t.row[i] * A.ldy + (t.head[i] * HQ_TILE + c0), A.y_bf16, v);
  }
}

// ----------------------------------------------------------------- attention
// One workgroup takes one KV head of one sequence and a run of its tokens (a
// chunk), each wave 32 tokens at a time.  Both products run on the matrix cores in
// bf16, which holds every code of the three formats exactly; the query and the
// weights enter as three bf16 terms each (8 + 8 + 8 bits, by truncation: their sum is
// the fp32 value itself), so the sums are fp32 sums.
//   scores   C[token, head] = K (16 tokens x 128) Q^T (16 heads, the group's G of them
//            used): lane l holds tokens 4 (l / 16) + r of head l % 16
//   values   O^T[dim, head] += V^T (16 dims x 32 tokens) P^T: with the 32 tokens of a step
//            numbered so that lane group l / 16 holds tokens 4 (l / 16) + 0 .. 3 of both
//            score tiles, the scores' C layout is P^T's operand layout, and no weight
//            moves between lanes.
// The head stays lane l % 16 throughout, so the softmax's maximum and sum are a
// lane's own but for two moves across the lane groups.
// Every code and scale is read once, so memory bounds it: 16 x 8192 tokens of int8, 8 KV
// heads (277 MB), take 54.4 us without the join (5.1 TB/s, a large copy's rate), 50.1 of them
// the loads alone; MXFP4 (143 MB) 35.7 with it, its conversions nearly as long as its loads.
// Below about 40 MB the chain from lengths over block ids and tokens to the end, 5.5 us, and
// the join's launch weigh more.

__device__ __forceinline__ v4_t mfma_bf16(const uint32_t* a, const uint32_t* b, v4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b_t, (v4w_t){a[0], a[1], a[2], a[3]}),
                                                 __builtin_bit_cast(v8b_t, (v4w_t){b[0], b[1], b[2], b[3]}), c, 0,
                                                 0, 0);
}

// v as three bf16 terms (as fp32 bit patterns whose low halves do not matter).
__device__ __forceinline__ void three_terms(float v, uint32_t* t) {
  t[0] = __float_as_uint(v);
  const float r = v - __uint_as_float(t[0] & 0xFFFF0000u);
  t[1] = __float_as_uint(r);
  t[2] = __float_as_uint(r - __uint_as_float(t[1] & 0xFFFF0000u));
}

// One word's codes as bf16 pairs: int8 and E4M3 two pairs from four codes, MXFP4
// four from eight (times 2^(byte - 127), `f` that factor).
template <int FMT>
__device__ __forceinline__ void pairs_of(uint32_t w, float f, uint32_t* o) {
  if constexpr (FMT == kInt8) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint((float)(int8_t)(w >> (8 * i)));
    o[0] = high_pair(x[0], x[1]);
    o[1] = high_pair(x[2], x[3]);
  } else if constexpr (FMT == kE4M3) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3));
  }
}

// The items of more than HQ_CACHE_UNPLANNED sequences, in one workgroup.  (1024 sequences
// of about 900 tokens, 8 KV heads in int8, take 335 us; 474 with every wave going through
// all lengths.)
constexpr int kPlanThreads = 1024;
template <int MODE>
__global__ __launch_bounds__(kPlanThreads) void hq_cache_plan_kernel(hq_cache_attn_args A) {
  __shared__ uint64_t s_sum[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // over the workgroup; every thread gets it
  auto sum = [&](uint64_t x) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m, 64);
    __syncthreads();  // the last sum has been read
    if (lane == 0) s_sum[wave] = x;
    __syncthreads();
    x = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) x += s_sum[i];
    return x;
  };
  auto seen = [&](int64_t i, bool tell, int32_t& tiles) {
    const CacheSpan of = cache_span_of<MODE>(A, i, tell);
    tiles = cache_tiles<MODE>(A, of.rows);
    return MODE == kAll ? of.len : of.seen();
  };
  int32_t tiles = 1;
  int64_t total = 0;
  for (int64_t i = tid; i < A.batch; i += kPlanThreads) {
    const int64_t len = seen(i, true, tiles);
    total += len * tiles;
  }
  total = (int64_t)sum((uint64_t)total);
  // it counts chunks for few sequences only: at most one per thread
  static_assert(HQ_CACHE_WG_TARGET + HQ_CACHE_WG_TARGET / 32 <= kPlanThreads, "");
  const int32_t mine = tid < A.batch ? seen(tid, false, tiles) : -1;
  const uint32_t chunk = cache_chunk(A, total, mine, tiles, [&](uint32_t n) { return (int64_t)sum(n); });
  uint64_t base = 0;  // items, and from bit 32 on split sequences, before these
  for (int64_t i0 = 0; i0 < A.batch; i0 += kPlanThreads) {
    const int64_t i = i0 + tid;
    const uint32_t n = i < A.batch ? cache_parts(seen(i, false, tiles), chunk) : 0u, split = n > 1;
    uint32_t items = n * (uint32_t)tiles, splits = split;
    wave_scan_incl2(items, splits);
    __syncthreads();  // the last sums have been read
    if (lane == 63) s_sum[wave] = (uint64_t)splits << 32 | items;
    __syncthreads();
    uint64_t at = base + ((uint64_t)(splits - split) << 32 | (items - n * (uint32_t)tiles));
    for (int x = 0; x < kPlanThreads / 64; ++x) {
      if (x < wave) at += s_sum[x];
      base += s_sum[x];
    }
    if (i < A.batch) A.parts[i] = {(int32_t)(uint32_t)at, (int32_t)n};
    // (a length that changes meanwhile could make them more than the table holds)
    if (split && (int64_t)(at >> 32) < A.joins) A.split[at >> 32] = (int32_t)i;
  }
  if (tid == 0) A.split[A.joins] = (int32_t)(base >> 32);
}

// The state that a wave carries over its tokens: per lane the maximum and sum of
// its column's scores, and the values' sum, acc[j][r] dim 8 (4 (l / 16) + r) + j.
struct CacheState {
  float m, l;
  v4_t acc[8];
};

// One step: 32 tokens' scores, the running maximum and sum, their values' sum.
// A head has C of the 16 columns, for the three terms of its query and weights: C = 4 (up
// to four heads) a column per term and one of zeros, in one product; C = 2 (up to eight)
// the first two in one product and the third beside zeros in another; C = 1 three products.
// (16 x 8192 tokens of MXFP4, 8 query heads per KV head: 40.0 us with two products, 42.2
// with three.)
template <int C>
constexpr int products() { return C == 4 ? 1 : C == 2 ? 2 : 3; }

template <int FMT, int C, typename WALK>
__device__ __forceinline__ void cache_step(CacheStep<FMT>& cur, const WALK& w, int32_t t, const typename WALK::Look& look,
                                           const uint32_t (&q)[products<C>()][4][4], int lane, CacheState& z) {
  constexpr int T = products<C>();
  const int n = lane & 15, g = lane >> 4;
  const bool cut = w.cut(look);
  auto dead = [&](int h, int r) { return w.dead(look, t, h, 4 * g + r); };
  if (cut) {
    // stale or absent tokens: their value codes count as zeros (their weight is
    // zero, but a stale code or scale may be a NaN)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (dead(h, r)) {
#pragma unroll
          for (int i = 0; i < CacheStep<FMT>::VW; ++i) cur.v[h][r][i] = 0u;
          cur.ks[h][r] = cur.vs[h][r] = 0.0f;
          cur.vx[h][r] = 0x7F7F7F7Fu;
        }
  }
  float p[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float f = FMT == kMx ? __uint_as_float(cur.kx[h] << 23) : 1.0f;
    constexpr int S = C == 1 ? T : 1;  // sums: columns of a head share one
    v4_t c[S];
#pragma unroll
    for (int i = 0; i < S; ++i) c[i] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint32_t a[4];
      if constexpr (FMT == kMx) {
        pairs_of<FMT>(cur.k[h][s], f, a);
      } else {
        pairs_of<FMT>(cur.k[h][2 * s], f, a);
        pairs_of<FMT>(cur.k[h][2 * s + 1], f, a + 2);
      }
#pragma unroll
      for (int i = T - 1; i >= 0; --i) c[i % S] = mfma_bf16(a, q[i][s], c[i % S]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = C == 1 ? c[0][r] + (c[S / 2][r] + c[S - 1][r]) : c[0][r];
      // the terms' sum, in each of the head's lanes
      if constexpr (C >= 2) x += dpp_xor<1>(x);
      if constexpr (C == 4) x += dpp_xor<2>(x);
      p[h][r] = FMT == kMx ? x : x * cur.ks[h][r];
    }
  }
  if (cut) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (dead(h, r)) p[h][r] = -__builtin_inff();
  }
  // a NaN stays one: it makes the head's outputs NaN
  float top = p[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = __builtin_elementwise_maximum(top, p[i >> 2][i & 3]);
  top = groups_max(top);
  if (__ballot(top > z.m)) {  // some column has a new maximum: all sums move to theirs
    const float mn = __builtin_fmaxf(z.m, top);
    const float alpha = __builtin_amdgcn_exp2f(z.m - (mn == -__builtin_inff() ? 0.0f : mn));
    z.m = mn;
    z.l *= alpha;
#pragma unroll
    for (int j = 0; j < 8; ++j) z.acc[j] *= alpha;
  }
  const float ref = z.m == -__builtin_inff() ? 0.0f : z.m;  // nothing seen yet
  uint32_t pt[T][4];  // the weights' terms: k index 4 h + r
  const uint32_t cut1 = (n & 3) < 1 ? 0u : 0xFFFF0000u, cut2 = (n & 3) < 2 ? 0u : 0xFFFF0000u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t tt[4][T];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(p[h][r] - ref);
      z.l += e;
      const float x = FMT == kMx ? e : e * cur.vs[h][r];
      if constexpr (C == 4) {  // the column's own term
        const float y = x - __uint_as_float(__float_as_uint(x) & cut1);
        tt[r][0] = __float_as_uint(y - __uint_as_float(__float_as_uint(y) & cut2));
      } else if constexpr (C == 2) {
        uint32_t t[3];
        three_terms(x, t);
        tt[r][0] = n & 1 ? t[1] : t[0];
        tt[r][1] = n & 1 ? 0u : t[2];
      } else {
        three_terms(x, tt[r]);
      }
    }
#pragma unroll
    for (int i = 0; i < T; ++i) {
      pt[i][2 * h] = high_pair(tt[0][i], tt[1][i]);
      pt[i][2 * h + 1] = high_pair(tt[2][i], tt[3][i]);
    }
  }
  // value codes: per token words of two dims, then per dim the tokens' pairs
#pragma unroll
  for (int w = 0; w < CacheStep<FMT>::VW; ++w) {
    constexpr int D = 4 / CacheStep<FMT>::VW;  // pairs of dims in a word
    uint32_t vf[2 * D][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        uint32_t x[2][D];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          pairs_of<FMT>(cur.v[h][r + e][w],
                        FMT == kMx ? __uint_as_float(((cur.vx[h][r + e] >> (8 * (n >> 2))) & 0xFFu) << 23) : 1.0f, x[e]);
#pragma unroll
        for (int d = 0; d < D; ++d) {
          vf[2 * d][2 * h + r / 2] = __builtin_amdgcn_perm(x[1][d], x[0][d], 0x05040100u);
          vf[2 * d + 1][2 * h + r / 2] = high_pair(x[0][d], x[1][d]);
        }
      }
#pragma unroll
    for (int i = T - 1; i >= 0; --i)
#pragma unroll
      for (int j = 0; j < 2 * D; ++j) z.acc[2 * D * w + j] = mfma_bf16(vf[j], pt[i], z.acc[2 * D * w + j]);
  }
}

template <int FMT, int C, int WAVES, int MODE>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void hq_cache_attn_kernel(
    hq_cache_attn_args A) {
  using R = CacheRing<FMT>;
  constexpr int HEADS = 16 / C, T = products<C>();
  extern __shared__ __attribute__((aligned(16))) uint8_t s_ring[];  // a wave's ring after the other
  __shared__ float s_m[WAVES][HEADS], s_l[WAVES][HEADS];
  // term i of the query lies in the second step of wave i's ring until that is first
  // loaded, a wave's sums in its own ring at the end
  static_assert(16 * kQPitch * sizeof(uint16_t) <= R::STEP && HEADS * kOPitch * sizeof(float) <= R::WAVE, "");
  auto q_row = [&](int term, int row) { return (uint16_t*)(s_ring + term * R::WAVE + R::STEP) + row * kQPitch; };
  auto o_row = [&](int w, int row) { return (float*)(s_ring + w * R::WAVE) + row * kOPitch; };
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4, grp = tid >> 4;
  const int wave = (int)readfirst((uint32_t)(tid >> 6));
  const int32_t j = (int32_t)(blockIdx.x / (uint32_t)A.heads_kv);
  const int32_t head = (int32_t)(blockIdx.x - (uint32_t)j * (uint32_t)A.heads_kv);
  const int32_t G = A.group, c0 = n * 8;
  Raw8 qraw = {};
  uint4 qd = {};
  auto load_query = [&](int32_t b) {
    if (grp < G) {
      qraw = load_raw8(A.q, ((int64_t)b * A.heads_q + (int64_t)head * G + grp) * HQ_TILE + c0, A.q_bf16);
      qd = sign_words(A.k_dsign16, head * HQ_TILE + c0);
    }
  };
  // A call that splits nothing knows its sequence: the whole table row (64 blocks at most)
  // and the query are on their way while the length is.  (8 of 1000 tokens: 11.1 us, 11.6.)
  // Where a window's blocks lie in the row goes by the length.
  int32_t ids = 0;
  if (!A.join && j < A.batch) {
    static_assert(HQ_CACHE_WHOLE <= 64 * 16, "");
    if (MODE == kAll) ids = A.table[(int64_t)j * A.max_blocks + min(lane, A.max_blocks - 1)];
    load_query(j);
  }
  const CacheItem it = cache_item<MODE>(A, j, lane, blockIdx.x == 0 && wave == 0);
  if (it.b < 0) return;
  // what the join goes by
  if (A.join && A.batch <= HQ_CACHE_UNPLANNED && j == it.first && head == 0 && tid == 0)
    A.parts[it.b] = {it.first, it.n};
  const int64_t pair0 = (int64_t)it.b * A.heads_q + (int64_t)head * G;
  const int32_t seen = MODE == kAll ? it.span.len : it.span.seen();
  if (seen == 0) {
    const float zero[8] = {};
    if (grp < G) store8(A.out, (pair0 + grp) * HQ_TILE + c0, A.out_bf16, zero);
    return;
  }
  // the chunk's steps of 32 tokens shared out over the waves
  const int32_t begin0 = (int32_t)(it.at * it.chunk), tokens = min(it.chunk, seen - begin0);
  const int32_t per = (tokens + 32 * WAVES - 1) / (32 * WAVES) * 32;
  const int32_t end = begin0 + min(tokens, (wave + 1) * per), begin = min(begin0 + wave * per, end);
  using Walk = std::conditional_t<MODE == kAll, CacheWalk, SpanWalk>;
  Walk w;
  w.start(A, it, head, begin);
  if (A.join || MODE != kAll) {
    w.ask(A, begin, lane);
    if (A.join) load_query(it.b);
  } else {
    w.first = 0;
    w.ids = ids;
  }
  w.got();
  w.template enter<FMT, true>(A, lane);
  uint8_t* ring = s_ring + wave * R::WAVE;
  typename Walk::Look sees = {}, next = {};
  if (begin < end) sees = w.template fetch<FMT>(A, begin, end, lane, ring);
  // ---- the query into the cache's coordinates, as three bf16 terms
  if (grp < HEADS) {
    float qv[8];
    expand8(qraw, A.q_bf16, qv);
    flip8(qv, qd);
    const XSigns sg(lane);
    fwht128(qv, sg);
    uint32_t t[8][3];
#pragma unroll
    for (int i = 0; i < 8; ++i) three_terms(qv[i] * A.qscale, t[i]);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint4 o;
      o.x = high_pair(t[0][i], t[1][i]);
      o.y = high_pair(t[2][i], t[3][i]);
      o.z = high_pair(t[4][i], t[5][i]);
      o.w = high_pair(t[6][i], t[7][i]);
      *(uint4*)(q_row(C == 4 ? 0 : C == 2 ? i >> 1 : i, C * grp + (C == 4 ? i : C == 2 ? i & 1 : 0)) + c0) = o;
    }
    if (C > 1) *(uint4*)(q_row(C == 4 ? 0 : 1, C * grp + C - 1) + c0) = make_uint4(0u, 0u, 0u, 0u);
  }
  __syncthreads();
  // step s of the contraction takes dims 32 (l / 16) + 8 s + j in lane l (the codes
  // that the lane's one run of 32 holds)
  uint32_t q[T][4][4];
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 x = *(const uint4*)(q_row(i, n) + 32 * g + 8 * s);
      q[i][s][0] = x.x; q[i][s][1] = x.y; q[i][s][2] = x.z; q[i][s][3] = x.w;
    }
  __syncthreads();  // the query's place is loaded over

  CacheState z;
  z.m = -__builtin_inff();
  z.l = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) z.acc[i] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
  if (begin + 32 < end) next = w.template fetch<FMT>(A, begin + 32, end, lane, ring + R::STEP);
  int32_t slot = 0;
  for (int32_t t = begin; t < end; t += 32) {
    // the loads of this step are done when at most the next step's are not
    if (t + 32 < end)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R::LOADS) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    CacheStep<FMT> cur;
    cache_take<FMT>(ring + slot * R::STEP, lane, cur);
    const typename Walk::Look here = sees;
    sees = next;
    if (t + 64 < end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what the ring held is in registers
      next = w.template fetch<FMT>(A, t + 64, end, lane, ring + slot * R::STEP);
    }
    slot ^= 1;
    cache_step<FMT, C>(cur, w, t, here, q, lane, z);
  }
  z.l = groups_sum(z.l);
  // ---- the waves' sums under one maximum, one head per 16 lanes
  // the head's columns together (with four, the last one's weights were a term over again),
  // its rows written by each of its lanes in turn
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = C == 4 && (n & 3) == 3 ? 0.0f : z.acc[i][r];
      if constexpr (C >= 2) x[i] += dpp_xor<1>(x[i]);
      if constexpr (C == 4) x[i] += dpp_xor<2>(x[i]);
    }
    if (n % C == r % C) {
      float* o = o_row(wave, n / C) + (4 * g + r) * 8;
      *(float4*)o = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)(o + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
  }
  if (g == 0 && n % C == 0) {
    s_m[wave][n / C] = z.m;
    s_l[wave][n / C] = z.l;
  }
  __syncthreads();
  if (grp >= G) return;
  float M = s_m[0][grp], L = 0.0f, v[8] = {};
#pragma unroll
  for (int x = 1; x < WAVES; ++x) M = __builtin_fmaxf(M, s_m[x][grp]);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
#pragma unroll
  for (int x = 0; x < WAVES; ++x) {
    const float f = __builtin_amdgcn_exp2f(s_m[x][grp] - ref);
    L = __builtin_fmaf(f, s_l[x][grp], L);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(f, o_row(x, grp)[c0 + i], v[i]);
  }
  if (it.n > 1) {
    const int64_t part = ((int64_t)j * A.heads_kv + head) * G + grp;
    store8(A.part_acc, part * HQ_TILE + c0, false, v);
    if (n == 0) {
      A.part_m[part] = M;
      A.part_l[part] = L;
    }
    return;
  }
  cache_finish(A, L, v, head, lane);
  store8(A.out, (pair0 + grp) * HQ_TILE + c0, A.out_bf16, v);
}

// Joins a query head's chunks under one maximum, in order, and moves the result
// back: one workgroup per query head, 16 lanes per chunk, for every sequence by its index;
// of a planned call only for the split ones (4096 sequences of about 100 tokens, 32 query
// heads: 416 us so, 478 with a workgroup for each).
__global__ __launch_bounds__(256) void hq_cache_join_kernel(hq_cache_attn_args A) {
  __shared__ float s_red[16];
  __shared__ float4 s_acc[16][32];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, grp = tid >> 4, c0 = n * 8;
  int64_t b = blockIdx.x / (uint32_t)A.heads_q;
  const int32_t hq = (int32_t)(blockIdx.x - (uint32_t)b * (uint32_t)A.heads_q), head = hq / A.group;
  if (A.batch > HQ_CACHE_UNPLANNED) {
    if (b >= A.split[A.joins]) return;
    b = A.split[b];
  }
  const hq_cache_of has = A.parts[b];
  const int32_t parts = has.n;
  if (parts == 1) return;  // already whole
  const int64_t part0 = ((int64_t)has.first * A.heads_kv + head) * A.group + (hq - head * A.group);
  // a group's first four chunks are loaded whole before the maxima meet
  float M = -__builtin_inff(), m[4], l[4], a[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int32_t x = grp + 16 * i;
    m[i] = M;
    l[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[i][e] = 0.0f;
    if (x >= parts) continue;
    const int64_t part = part0 + (int64_t)x * A.heads_q;
    m[i] = A.part_m[part];
    l[i] = A.part_l[part];
    load8(A.part_acc, part * HQ_TILE + c0, false, a[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) M = __builtin_fmaxf(M, m[i]);
  for (int32_t x = grp + 64; x < parts; x += 16) M = __builtin_fmaxf(M, A.part_m[part0 + (int64_t)x * A.heads_q]);
  if (n == 0) s_red[grp] = M;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 16; ++k) M = __builtin_fmaxf(M, s_red[k]);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
  float L = 0.0f, v[8] = {};
  auto add = [&](float mx, float lx, const float* ax) {
    const float f = __builtin_amdgcn_exp2f(mx - ref);
    L = __builtin_fmaf(f, lx, L);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(f, ax[e], v[e]);
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) add(m[i], l[i], a[i]);
  for (int32_t x = grp + 64; x < parts; x += 16) {
    const int64_t part = part0 + (int64_t)x * A.heads_q;
    float ax[8];
    load8(A.part_acc, part * HQ_TILE + c0, false, ax);
    add(A.part_m[part], A.part_l[part], ax);
  }
  __syncthreads();  // every group has read s_red
  s_acc[grp][2 * n] = make_float4(v[0], v[1], v[2], v[3]);
  s_acc[grp][2 * n + 1] = make_float4(v[4], v[5], v[6], v[7]);
  if (n == 0) s_red[grp] = L;
  __syncthreads();
  if (tid >= 16) return;  // group 0 finishes: no barrier follows
  L = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.0f;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const float4 x = s_acc[k][2 * n], y = s_acc[k][2 * n + 1];
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
    L += s_red[k];
  }
  cache_finish(A, L, v, head, lane);
  store8(A.out, (b * A.heads_q + hq) * HQ_TILE + c0, A.out_bf16, v);
}

}  // namespace

#define HQ_CACHE_FORMATS(KERNEL, FMT, GRID, STREAM, ARGS)                                        \
  switch (FMT) {                                                                                 \
    case HQ_INT8: hipLaunchKernelGGL(KERNEL<kInt8>, GRID, dim3(256), 0, STREAM, ARGS); break;    \
    case HQ_E4M3: hipLaunchKernelGGL(KERNEL<kE4M3>, GRID, dim3(256), 0, STREAM, ARGS); break;    \
    default: hipLaunchKernelGGL(KERNEL<kMx>, GRID, dim3(256), 0, STREAM, ARGS);                  \
  }

int hq_launch_cache_write(const hq_cache_io_args& a, int format, int sides, void* stream) {
  const dim3 grid((a.tiles + kIoTiles - 1) / kIoTiles, (uint32_t)sides);
  HQ_CACHE_FORMATS(hq_cache_write_kernel, format, grid, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

int hq_launch_cache_read(const hq_cache_io_args& a, int format, void* stream) {
  const dim3 grid((a.tiles + kIoTiles - 1) / kIoTiles);
  HQ_CACHE_FORMATS(hq_cache_read_kernel, format, grid, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

template <int FMT, int C, int WAVES, int MODE>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  static hq_lds_granted granted;
  constexpr size_t lds = (size_t)WAVES * CacheRing<FMT>::WAVE;
  if (const int e = hq_allow_lds((const void*)hq_cache_attn_kernel<FMT, C, WAVES, MODE>, lds, granted)) return e;
  hipLaunchKernelGGL((hq_cache_attn_kernel<FMT, C, WAVES, MODE>), grid, dim3(64 * WAVES), lds, st, a);
  return 0;
}

// Calls that leave half the CUs without a workgroup have eight waves share its tokens.
// (8 KV heads in E4M3: one sequence of 1000 tokens takes 10.6 us, 12.3 with four waves, 16 of
// them 12.2 and 13.3; but 32 of 300, on every CU, 10.9 and 9.8.)
template <int FMT, int C, int MODE>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  return grid.x <= 128 ? launch_attn<FMT, C, 2 * HQ_CACHE_WAVES, MODE>(a, grid, st)
                       : launch_attn<FMT, C, HQ_CACHE_WAVES, MODE>(a, grid, st);
}

template <int FMT, int MODE>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  return a.group <= 4   ? launch_attn<FMT, 4, MODE>(a, grid, st)
         : a.group <= 8 ? launch_attn<FMT, 2, MODE>(a, grid, st)
                        : launch_attn<FMT, 1, MODE>(a, grid, st);
}

void hq_launch_cache_plan(const hq_cache_attn_args& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const dim3 one(1), wg(kPlanThreads);
  if (a.starts)
    hipLaunchKernelGGL(hq_cache_plan_kernel<kTree>, one, wg, 0, st, a);
  else if (a.window)
    hipLaunchKernelGGL(hq_cache_plan_kernel<kWindow>, one, wg, 0, st, a);
  else
    hipLaunchKernelGGL(hq_cache_plan_kernel<kAll>, one, wg, 0, st, a);
}

template <int MODE>
static int launch_attn(const hq_cache_attn_args& a, int format, hipStream_t st) {
  const dim3 grid((uint32_t)(a.items * a.heads_kv)), wg(256);
  int e = 0;
  if (a.join && a.batch > HQ_CACHE_UNPLANNED) hq_launch_cache_plan(a, st);
  switch (format) {
    case HQ_INT8: e = launch_attn<kInt8, MODE>(a, grid, st); break;
    case HQ_E4M3: e = launch_attn<kE4M3, MODE>(a, grid, st); break;
    default: e = launch_attn<kMx, MODE>(a, grid, st);
  }
  if (e) return e;
  if (a.join && a.joins)
    hipLaunchKernelGGL(hq_cache_join_kernel, dim3((uint32_t)(a.joins * a.heads_q)), wg, 0, st, a);
  return (int)hipGetLastError();
}

int hq_launch_cache_attention(const hq_cache_attn_args& a, int format, void* stream) {
  return a.window ? launch_attn<kWindow>(a, format, (hipStream_t)stream)
                  : launch_attn<kAll>(a, format, (hipStream_t)stream);
}
