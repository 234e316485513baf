// gfx950 kernels of the fixed-rate key-value cache: rows cast into slots
// (hq_cache_write), read back (hq_cache_read), and one query token per sequence
// attending over a paged cache (hq_cache_attention).
//
// A stored head vector is the cast of y = H D x (H the 128-point Sylvester
// matrix, D the plan's signs of the head's columns): int8 or E4M3 codes c with one
// fp32 scale s, y = s c, or MXFP4.  H D / sqrt(128) is orthogonal, so
//   q . x = (H D q) . y / 128     and     sum_t p_t x_t = D H (sum_t p_t y_t) / 128:
// the attention moves each query once and each output back once, and works on
// the codes as they lie.  Rows lie as [block, head, token of the block], so one head's
// tokens of a block are one run of memory.
#include <hip/hip_runtime.h>

#include "hq_device.h"
#include "hq_lds.h"

#pragma clang fp contract(off)

namespace {

typedef float v2f_t __attribute__((ext_vector_type(2)));

constexpr int kInt8 = HQ_INT8, kE4M3 = HQ_E4M3, kMx = HQ_MXFP4;

template <int FMT>
constexpr int row_bytes() { return FMT == kMx ? HQ_TILE / 2 : HQ_TILE; }

// 8 consecutive values (16-byte aligned) of a bf16 or fp32 array as fp32.
__device__ __forceinline__ void load8(const void* p, int64_t i, bool bf16, float* v) {
  if (bf16) {
    const uint4 raw = *(const uint4*)((const uint16_t*)p + i);
    const uint32_t w4[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = bf16_to_f32(w4[k] & 0xFFFFu);
      v[2 * k + 1] = __uint_as_float(w4[k] & 0xFFFF0000u);
    }
  } else {
    const float4 a = *(const float4*)((const float*)p + i);
    const float4 b = *(const float4*)((const float*)p + i + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

// The same in two steps, so that other loads start between them.  The loads have no
// branch, whose end would wait for them: of bf16 the second takes the first's words again.
struct Raw8 {
  uint4 a, b;
};
__device__ __forceinline__ Raw8 load_raw8(const void* p, int64_t i, bool bf16) {
  const uint8_t* at = (const uint8_t*)p + (bf16 ? 2 * i : 4 * i);
  return {*(const uint4*)at, *(const uint4*)(at + (bf16 ? 0 : 16))};
}
__device__ __forceinline__ void expand8(const Raw8& r, bool bf16, float* v) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    v[k] = __uint_as_float(!bf16 ? w[k] : k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
}

__device__ __forceinline__ void store8(void* p, int64_t i, bool bf16, const float* v) {
  if (bf16) {
    uint4 o;
    o.x = cvt_pk_bf16(v[0], v[1]);
    o.y = cvt_pk_bf16(v[2], v[3]);
    o.z = cvt_pk_bf16(v[4], v[5]);
    o.w = cvt_pk_bf16(v[6], v[7]);
    *(uint4*)((uint16_t*)p + i) = o;
  } else {
    float* o = (float*)p + i;
    *(float4*)o = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// D of the 8 columns from col on, as bf16 sign bits per pair of columns.
__device__ __forceinline__ uint4 sign_words(const uint32_t* dsign16, int64_t col) {
  return *(const uint4*)(dsign16 + (col >> 1));
}

__device__ __forceinline__ void flip8(float* v, uint4 d) {
  const uint32_t w[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = xor_sign(v[2 * i], w[i] << 16);
    v[2 * i + 1] = xor_sign(v[2 * i + 1], w[i] & 0xFFFF0000u);
  }
}

// a / b for a constant b, correctly rounded where nothing underflows: the quotient
// by the rounded reciprocal, corrected by its exact remainder.
__device__ __forceinline__ float over(float a, float b) {
  const float r = 1.0f / b, q = a * r;
  return __builtin_fmaf(__builtin_fmaf(-b, q, a), r, q);
}

__device__ __forceinline__ void report(hq_stats* s, int32_t err) {
  if (s) atomicCAS(&s->status, 0u, (uint32_t)err);
}

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
    float am = amax_or_nan<8>(v[i]);
    am = __builtin_elementwise_maximum(am, dpp_xor<1>(am));
    am = __builtin_elementwise_maximum(am, dpp_xor<2>(am));
    am = __builtin_elementwise_maximum(am, swz_xor4(am));
    am = __builtin_elementwise_maximum(am, dpp_xor<8>(am));
    // a vector with an infinite or NaN value has no scale: codes 0, scale NaN
    const bool bad = !(am <= 3.4028234663852886e38f);
    if (__builtin_expect(bad, 0)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
      if (live && (lane & 15) == 0 && S.stats) {
        atomicAdd(&S.stats->overflow_tiles, 1u);
        report(S.stats, HQ_ERR_OVERFLOW);
      }
    }
    if constexpr (FMT == kMx) {
      int32_t X;
      const uint32_t packed = mxfp4_x8(v[i], X) ^ (sg.sigma ? 0x88888888u : 0u);
      if (!live) continue;
      *(uint32_t*)(S.codes + vec * row_bytes<FMT>() + c0 / 2) = packed;
      if ((lane & 3) == 0) ((uint8_t*)S.scales)[vec * 4 + ((lane & 15) >> 2)] = bad ? 0xFFu : (uint8_t)(X + 127);
    } else {
      constexpr float top = FMT == kE4M3 ? 448.0f : 127.0f;
      // below 2^-100 the reciprocal could overflow: such a vector is stored as zeros
      const bool zero = bad || am < 0x1p-100f;
      const float inv = zero ? 0.0f : xor_sign(top / am, sg.sigma);
      // |q| is top (1 + 2^-23) at most, which rounds to top in both formats: no clamp
      uint2 packed;
      if constexpr (FMT == kE4M3) {
        packed.x = e4m3x4(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
        packed.y = e4m3x4(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
      } else {
        packed = int8x8(v[i], inv);
      }
      if (!live) continue;
      *(uint2*)(S.codes + vec * row_bytes<FMT>() + c0) = packed;
      if ((lane & 15) == 0) ((float*)S.scales)[vec] = bad ? __builtin_nanf("") : zero ? 0.0f : over(am, top);
    }
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
typedef float v4_t __attribute__((ext_vector_type(4)));
typedef __bf16 v8b_t __attribute__((ext_vector_type(8)));
typedef uint32_t v4w_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4_t mfma_bf16(const uint32_t* a, const uint32_t* b, v4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b_t, (v4w_t){a[0], a[1], a[2], a[3]}),
                                                 __builtin_bit_cast(v8b_t, (v4w_t){b[0], b[1], b[2], b[3]}), c, 0,
                                                 0, 0);
}

// The high halves of two words: two bf16 from two fp32 by truncation, lo first.
__device__ __forceinline__ uint32_t high_pair(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
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

// Maximum and sum over the four lane groups (lanes l, l ^ 16, l ^ 32, l ^ 48): a swap
// of a value with itself leaves the two halves (or row pairs) side by side.
typedef uint32_t v2u_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float groups_max(float x) {
  const v2u_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const v2u_t b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  const v2u_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const v2u_t b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---- who does what
// The tokens of a call are cut into chunks of about one length, as many workgroups
// as the chip holds at once over all sequences and KV heads, so that a batch of uneven
// lengths keeps it as busy as an even one.  Item j is chunk j - first of sequence b.
// Up to HQ_CACHE_UNPLANNED sequences every wave finds its item by itself, one length per
// lane; more are planned by a launch before (hq_cache_plan_kernel), whose table the waves
// search.
constexpr int32_t kStep = 32 * HQ_CACHE_WAVES;
struct CacheItem {
  int32_t b;       // -1: behind the last item
  int32_t n;       // chunks of this sequence (an empty one has one, which writes its zeros)
  int32_t first;   // the sequence's first item
  int32_t len, chunk;
};

__device__ __forceinline__ int32_t cache_len(const hq_cache_attn_args& A, int64_t b, bool tell) {
  const int64_t cap = (int64_t)A.max_blocks * A.block_tokens;
  const int64_t len = A.seq_lens[b];
  if (len >= 0 && len <= cap) return (int32_t)len;
  if (tell) report(A.stats, HQ_ERR_INVALID_ARG);
  return len < 0 ? 0 : (int32_t)cap;
}

__device__ __forceinline__ uint32_t cache_parts(int32_t len, uint32_t chunk) {
  return len == 0 ? 1u : ((uint32_t)len + chunk - 1) / chunk;
}

// The longest a chunk may be: whole steps of all waves, HQ_CACHE_LEAST tokens at
// least; one of 2^30 holds any sequence.  An even share of the workgroups aimed at
// would be right if every sequence were a multiple of it.  A sequence's last chunk is
// not, and what that adds opens a second round of workgroups, so the share grows by
// eighths until the chunks fit but for a few, to its double at most.  (24 sequences of
// up to 6001 tokens, 8 KV heads in E4M3: 560 chunks of the even share take 51.7 us, 528 of
// its 9 / 8 take 41.4.)  More sequences than that take several rounds in any case.
// `total`: all tokens; `mine`: a lane's or thread's own sequence's, -1 without one; `sum`
// adds a number over all of these.
template <typename SUM>
__device__ __forceinline__ uint32_t cache_chunk(const hq_cache_attn_args& A, int64_t total, int32_t mine, SUM sum) {
  const int64_t even = (total * A.heads_kv + HQ_CACHE_WG_TARGET - 1) / HQ_CACHE_WG_TARGET;
  const int64_t few = (HQ_CACHE_WG_TARGET + HQ_CACHE_WG_TARGET / 32) / A.heads_kv;
  uint32_t chunk = HQ_CACHE_LEAST;
  for (int e = 8; e <= 16; ++e) {
    const int64_t c = min(((even * e >> 3) + kStep - 1) & -(int64_t)kStep, (int64_t)1 << 30);
    chunk = max(chunk, readfirst((uint32_t)c));
    if (A.batch > few) break;
    // about: a length a hair over a multiple may count as the multiple
    const float per = __builtin_amdgcn_rcpf((float)chunk) * 0.999999f;
    if (sum(mine < 0 ? 0u : max(1u, (uint32_t)__builtin_ceilf((float)mine * per))) <= few) break;
  }
  return chunk;
}

// Whole steps of all waves, about as many in each of a sequence's n chunks.
__device__ __forceinline__ int32_t even_chunk(int32_t len, int32_t n) {
  return (len + n * kStep - 1) / (n * kStep) * kStep;
}

__device__ __forceinline__ CacheItem cache_item(const hq_cache_attn_args& A, int32_t j, int lane, bool tell) {
  CacheItem it;
  it.b = -1;
  if (!A.join) {  // one chunk each
    if (j >= A.batch) return it;
    it.b = it.first = j;
    it.n = 1;
    it.len = (int32_t)readfirst((uint32_t)cache_len(A, it.b, true));
    it.chunk = HQ_CACHE_WHOLE;
    return it;
  }
  if (A.batch > HQ_CACHE_UNPLANNED) {
    // the last sequence whose first item is j at most, 64 places a step
    int64_t lo = 0;
    for (int64_t span = A.batch; span > 1;) {
      const int64_t stride = (span + 63) >> 6, at = lo + lane * stride;
      const bool below = lane * stride < span && A.parts[at].first <= j;
      const int64_t last = __popcll(__ballot(below)) - 1;  // the first place is always below
      lo += last * stride;
      span = min(stride, span - last * stride);
    }
    const hq_cache_of of = A.parts[lo];
    it.first = (int32_t)readfirst((uint32_t)of.first);
    it.n = (int32_t)readfirst((uint32_t)of.n);
    if (j >= it.first + it.n) return it;
    it.b = (int32_t)readfirst((uint32_t)lo);
    it.len = (int32_t)readfirst((uint32_t)cache_len(A, it.b, false));
  } else {
    static_assert(HQ_CACHE_UNPLANNED <= 64, "");
    const bool in = lane < A.batch;
    const int32_t len = in ? cache_len(A, lane, tell) : -1;
    int64_t total = max(len, 0);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m, 64);
    const uint32_t chunk = cache_chunk(A, total, len, [](uint32_t n) { return wave_total(n); });
    const uint32_t n = in ? cache_parts(len, chunk) : 0u;
    const int32_t incl = (int32_t)wave_scan_incl(n);
    if (j >= __builtin_amdgcn_readlane(incl, 63)) return it;
    const int at = __popcll(__ballot(incl <= j));
    it.b = at;
    it.n = (int32_t)__builtin_amdgcn_readlane(n, at);
    it.first = __builtin_amdgcn_readlane(incl, at) - it.n;
    it.len = __builtin_amdgcn_readlane(len, at);
  }
  it.chunk = even_chunk(it.len, it.n);
  return it;
}

// The items of more than HQ_CACHE_UNPLANNED sequences, in one workgroup.  (1024 sequences
// of about 900 tokens, 8 KV heads in int8, take 335 us; 474 with every wave going through
// all lengths.)
constexpr int kPlanThreads = 1024;
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
  int64_t total = 0;
  for (int64_t i = tid; i < A.batch; i += kPlanThreads) total += cache_len(A, i, true);
  total = (int64_t)sum((uint64_t)total);
  // it counts chunks for few sequences only: at most one per thread
  static_assert(HQ_CACHE_WG_TARGET + HQ_CACHE_WG_TARGET / 32 <= kPlanThreads, "");
  const uint32_t chunk = cache_chunk(A, total, tid < A.batch ? cache_len(A, tid, false) : -1,
                                     [&](uint32_t n) { return (int64_t)sum(n); });
  uint64_t base = 0;  // items, and from bit 32 on split sequences, before these
  for (int64_t i0 = 0; i0 < A.batch; i0 += kPlanThreads) {
    const int64_t i = i0 + tid;
    const uint32_t n = i < A.batch ? cache_parts(cache_len(A, i, false), chunk) : 0u, split = n > 1;
    uint32_t items = n, splits = split;
    wave_scan_incl2(items, splits);
    __syncthreads();  // the last sums have been read
    if (lane == 63) s_sum[wave] = (uint64_t)splits << 32 | items;
    __syncthreads();
    uint64_t at = base + ((uint64_t)(splits - split) << 32 | (items - n));
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

// ---- a wave's tokens
// A wave's tokens come through LDS, loaded there straight from memory (no register
// waits for them) in a ring of two steps of 32 tokens, each two halves of 16: the key
// codes, the value codes, and the 64 bytes of scales of each (256 with their copies).  A row's 16-byte chunks are
// permuted by its index, which the loads' source addresses do, so that the reads
// below meet no bank twice.
template <int FMT>
struct CacheRing {
  static constexpr int RB = row_bytes<FMT>();
  static constexpr int V = 16 * RB, SCALES = 32 * RB;      // places in a half
  static constexpr int HALF = SCALES + 512, STEP = 2 * HALF, WAVE = 2 * STEP;
  static constexpr int LOADS = 2 * (2 * (16 * RB / 1024) + 2);  // of a step
  // 16-byte chunk c of row r lies at chunk c ^ swizzle(r)
  static __device__ __forceinline__ uint32_t swizzle(uint32_t r) { return FMT == kMx ? (r >> 1) & 3 : r & 7; }
};

// One step's codes and scales in registers.
template <int FMT>
struct CacheStep {
  static constexpr int KW = FMT == kMx ? 4 : 8;  // words of 32 codes
  static constexpr int VW = FMT == kMx ? 1 : 2;  // words of 8 codes
  uint32_t k[2][KW];         // token 16 h + l % 16, dims 32 (l / 16) ..
  uint32_t v[2][4][VW];      // token 16 h + 4 (l / 16) + r, dims 8 (l % 16) ..
  float ks[2][4], vs[2][4];  // fp32 scales of those four tokens
  uint32_t kx[2], vx[2][4];  // MXFP4: the scale byte of k, the four bytes of v's tokens
};

typedef __attribute__((address_space(3))) void lds_void;

// A run of `bytes` from p on as a buffer resource (p the same in every lane).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t run_of(const void* p, int64_t at, uint32_t bytes) {
  const uint64_t a = (uint64_t)p + at;
  const uint64_t u = (uint64_t)readfirst((uint32_t)(a >> 32)) << 32 | readfirst((uint32_t)a);
  return __builtin_amdgcn_make_buffer_rsrc((void*)u, 0, bytes, 0x00020000);
}

// Where a wave stands in its sequence: token off of block blk of the table row, and
// that block's head as buffers.  The ids of 64 blocks ahead are one per lane, so that
// following the table costs a lane read and not a load that the next loads' addresses
// wait for.
struct CacheWalk {
  const int32_t* table;
  int32_t last;  // the sequence's last block
  int32_t head, blk, off;
  int32_t first, ids;  // lane l: block first + l
  __amdgpu_buffer_rsrc_t k, v, ks, vs;
  bool bad;  // the block lies outside the cache: its buffers are empty
  __device__ __forceinline__ void ask(int lane) {
    first = blk;
    ids = table[min(blk + lane, last)];
  }
  // the wait for it stands here: at its uses it would wait for the tokens in flight
  __device__ __forceinline__ void got() { asm volatile("" : "+v"(ids)); }
  template <int FMT, bool KNOWN>  // KNOWN: the ids are those of this block on
  __device__ __forceinline__ void enter(const hq_cache_attn_args& A, int lane) {
    if (!KNOWN && blk - first >= 64) {
      ask(lane);
      got();
    }
    const int32_t id = __builtin_amdgcn_readlane(ids, blk - first);
    bad = (uint32_t)id >= (uint32_t)A.blocks;
    if (bad && head == 0 && lane == 0) report(A.stats, HQ_ERR_INVALID_ARG);
    const uint32_t n = bad ? 0u : (uint32_t)A.block_tokens;
    const int64_t row = bad ? 0 : ((int64_t)id * A.heads_kv + head) * A.block_tokens;
    k = run_of(A.k_codes, row * row_bytes<FMT>(), n * row_bytes<FMT>());
    v = run_of(A.v_codes, row * row_bytes<FMT>(), n * row_bytes<FMT>());
    ks = run_of(A.k_scales, row * 4, n * 4);
    vs = run_of(A.v_scales, row * 4, n * 4);
  }
  // Starts the loads of the 32 tokens from t on into `step` (LDS) and moves the walk
  // past them; live[h]: tokens of each half to attend to.
  template <int FMT>
  __device__ __forceinline__ void fetch(const hq_cache_attn_args& A, int32_t t, int32_t end, int lane, uint8_t* step,
                                        int32_t (&live)[2]) {
    using R = CacheRing<FMT>;
    constexpr uint32_t RPL = 1024 / R::RB, CPR = R::RB / 16;  // rows of a load, chunks of a row
    const uint32_t row_in = lane / CPR, chunk = lane % CPR;
    const uint32_t from = row_in * R::RB + (chunk ^ R::swizzle(row_in)) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (t + 16 * h < end && off == A.block_tokens) {  // 16 divides a block
        off = 0;
        ++blk;
        enter<FMT, false>(A, lane);
      }
      // a half behind the end loads its block's first tokens, one of a block outside the
      // cache nothing (its buffers are empty), so that a step is always the same loads;
      // nothing reads them
      live[h] = bad ? 0 : min(max(end - t - 16 * h, 0), 16);
      const uint32_t at = live[h] ? off : 0;
      off += 16;
      uint8_t* to = step + h * R::HALF;
#pragma unroll
      for (uint32_t i = 0; i < 16 / RPL; ++i) {
        const uint32_t rows = at * R::RB + i * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(k, (lds_void*)(to + i * 1024), 16, from, rows, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(v, (lds_void*)(to + R::V + i * 1024), 16, from, rows, 0, 0);
      }
      const uint32_t token = (lane & 15) * 4;  // four times over
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ks, (lds_void*)(to + R::SCALES), 4, token, at * 4, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vs, (lds_void*)(to + R::SCALES + 256), 4, token, at * 4, 0, 0);
    }
  }
};

// A step's codes and scales out of LDS.
template <int FMT>
__device__ __forceinline__ void cache_take(const uint8_t* step, int lane, CacheStep<FMT>& s) {
  using R = CacheRing<FMT>;
  const uint32_t n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint8_t* half = step + h * R::HALF;
#pragma unroll
    for (int i = 0; i < CacheStep<FMT>::KW; i += 4) {
      const uint32_t chunk = (FMT == kMx ? g : 2 * g + i / 4) ^ R::swizzle(n);
      const uint4 x = *(const uint4*)(half + n * R::RB + chunk * 16);
      s.k[h][i] = x.x; s.k[h][i + 1] = x.y; s.k[h][i + 2] = x.z; s.k[h][i + 3] = x.w;
    }
    const uint8_t* sc = half + R::SCALES;
    if constexpr (FMT == kMx) {
      s.kx[h] = sc[4 * n + g];
      const uint4 x = *(const uint4*)(sc + 256 + 16 * g);
      s.vx[h][0] = x.x; s.vx[h][1] = x.y; s.vx[h][2] = x.z; s.vx[h][3] = x.w;
    } else {
      const float4 x = *(const float4*)(sc + 16 * g);
      const float4 y = *(const float4*)(sc + 256 + 16 * g);
      s.ks[h][0] = x.x; s.ks[h][1] = x.y; s.ks[h][2] = x.z; s.ks[h][3] = x.w;
      s.vs[h][0] = y.x; s.vs[h][1] = y.y; s.vs[h][2] = y.z; s.vs[h][3] = y.w;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t row = 4 * g + r;
      if constexpr (FMT == kMx) {
        s.v[h][r][0] = *(const uint32_t*)(half + R::V + row * R::RB + ((n >> 2) ^ R::swizzle(row)) * 16 + (n & 3) * 4);
      } else {
        const uint2 x = *(const uint2*)(half + R::V + row * R::RB + ((n >> 1) ^ R::swizzle(row)) * 16 + (n & 1) * 8);
        s.v[h][r][0] = x.x; s.v[h][r][1] = x.y;
      }
    }
  }
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

template <int FMT, int C>
__device__ __forceinline__ void cache_step(CacheStep<FMT>& cur, const int32_t (&live)[2],
                                           const uint32_t (&q)[products<C>()][4][4], int lane, CacheState& z) {
  constexpr int T = products<C>();
  const int n = lane & 15, g = lane >> 4;
  if (live[0] + live[1] < 32) {
    // stale or absent tokens: their value codes count as zeros (their weight is
    // zero, but a stale code or scale may be a NaN)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * g + r >= live[h]) {
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
  if (live[0] + live[1] < 32) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * g + r >= live[h]) p[h][r] = -__builtin_inff();
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

constexpr int kQPitch = HQ_TILE + 8;  // bf16 of a query row in LDS
constexpr int kOPitch = HQ_TILE + 4;  // floats of an output row in LDS

// v * 1 / (128 sum) moved back to the head's own coordinates.
__device__ __forceinline__ void cache_finish(const hq_cache_attn_args& A, float L, float* v, int32_t head, int lane) {
  const float inv = L == 0.0f ? 0.0f : 1.0f / (L * 128.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
  const XSigns sg(lane);
  fwht128(v, sg);
  flip8(v, sign_words(A.v_dsign16, head * HQ_TILE + (lane & 15) * 8));
}

template <int FMT, int C, int WAVES>
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
  int32_t ids = 0;
  if (!A.join && j < A.batch) {
    static_assert(HQ_CACHE_WHOLE <= 64 * 16, "");
    ids = A.table[(int64_t)j * A.max_blocks + min(lane, A.max_blocks - 1)];
    load_query(j);
  }
  const CacheItem it = cache_item(A, j, lane, blockIdx.x == 0 && wave == 0);
  if (it.b < 0) return;
  // what the join goes by
  if (A.join && A.batch <= HQ_CACHE_UNPLANNED && j == it.first && head == 0 && tid == 0)
    A.parts[it.b] = {it.first, it.n};
  const int64_t pair0 = (int64_t)it.b * A.heads_q + (int64_t)head * G;
  if (it.len == 0) {
    const float zero[8] = {};
    if (grp < G) store8(A.out, (pair0 + grp) * HQ_TILE + c0, A.out_bf16, zero);
    return;
  }
  // the chunk's steps of 32 tokens shared out over the waves
  const int32_t begin0 = (int32_t)((j - it.first) * it.chunk), tokens = min(it.chunk, it.len - begin0);
  const int32_t per = (tokens + 32 * WAVES - 1) / (32 * WAVES) * 32;
  const int32_t end = begin0 + min(tokens, (wave + 1) * per), begin = min(begin0 + wave * per, end);
  CacheWalk w;
  w.table = A.table + (int64_t)it.b * A.max_blocks;
  w.last = (it.len - 1) / A.block_tokens;
  w.head = head;
  w.blk = min(begin / A.block_tokens, w.last);
  w.off = begin - w.blk * A.block_tokens;
  if (A.join) {
    w.ask(lane);
    load_query(it.b);
  } else {
    w.first = 0;
    w.ids = ids;
  }
  w.got();
  w.enter<FMT, true>(A, lane);
  uint8_t* ring = s_ring + wave * R::WAVE;
  int32_t live[2], next[2] = {0, 0};
  if (begin < end) w.fetch<FMT>(A, begin, end, lane, ring, live);
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
  if (begin + 32 < end) w.fetch<FMT>(A, begin + 32, end, lane, ring + R::STEP, next);
  int32_t slot = 0;
  for (int32_t t = begin; t < end; t += 32) {
    // the loads of this step are done when at most the next step's are not
    if (t + 32 < end)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R::LOADS) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    CacheStep<FMT> cur;
    cache_take<FMT>(ring + slot * R::STEP, lane, cur);
    const int32_t here[2] = {live[0], live[1]};
    live[0] = next[0];
    live[1] = next[1];
    if (t + 64 < end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what the ring held is in registers
      w.fetch<FMT>(A, t + 64, end, lane, ring + slot * R::STEP, next);
    }
    slot ^= 1;
    cache_step<FMT, C>(cur, here, q, lane, z);
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

template <int FMT, int C, int WAVES>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  static hq_lds_granted granted;
  constexpr size_t lds = (size_t)WAVES * CacheRing<FMT>::WAVE;
  if (const int e = hq_allow_lds((const void*)hq_cache_attn_kernel<FMT, C, WAVES>, lds, granted)) return e;
  hipLaunchKernelGGL((hq_cache_attn_kernel<FMT, C, WAVES>), grid, dim3(64 * WAVES), lds, st, a);
  return 0;
}

// Calls that leave half the CUs without a workgroup have eight waves share its tokens.
// (8 KV heads in E4M3: one sequence of 1000 tokens takes 10.6 us, 12.3 with four waves, 16 of
// them 12.2 and 13.3; but 32 of 300, on every CU, 10.9 and 9.8.)
template <int FMT, int C>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  return grid.x <= 128 ? launch_attn<FMT, C, 2 * HQ_CACHE_WAVES>(a, grid, st)
                       : launch_attn<FMT, C, HQ_CACHE_WAVES>(a, grid, st);
}

template <int FMT>
static int launch_attn(const hq_cache_attn_args& a, dim3 grid, hipStream_t st) {
  return a.group <= 4   ? launch_attn<FMT, 4>(a, grid, st)
         : a.group <= 8 ? launch_attn<FMT, 2>(a, grid, st)
                        : launch_attn<FMT, 1>(a, grid, st);
}

int hq_launch_cache_attention(const hq_cache_attn_args& a, int format, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const dim3 grid((uint32_t)(a.items * a.heads_kv)), wg(256);
  int e = 0;
  if (a.join && a.batch > HQ_CACHE_UNPLANNED)
    hipLaunchKernelGGL(hq_cache_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
  switch (format) {
    case HQ_INT8: e = launch_attn<kInt8>(a, grid, st); break;
    case HQ_E4M3: e = launch_attn<kE4M3>(a, grid, st); break;
    default: e = launch_attn<kMx>(a, grid, st);
  }
  if (e) return e;
  if (a.join && a.joins)
    hipLaunchKernelGGL(hq_cache_join_kernel, dim3((uint32_t)(a.joins * a.heads_q)), wg, 0, st, a);
  return (int)hipGetLastError();
}
