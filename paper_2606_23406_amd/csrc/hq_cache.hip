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

__device__ __forceinline__ void report(hq_stats* s, int32_t err) {
  if (s) atomicCAS(&s->status, 0u, (uint32_t)err);
}

// ------------------------------------------------------------- write and read
// 16 lanes take one head vector, 8 values each; a wave four of them, neighbouring
// heads of one token where there are four.

struct CacheTile {
  int64_t row;   // token row of the call
  int32_t head;
  int64_t at;    // index of the stored head vector, or -1
};

__device__ __forceinline__ CacheTile cache_tile(const hq_cache_io_args& A, const hq_cache_side& S, int lane,
                                                bool first) {
  const uint32_t tile = blockIdx.x * 16u + (threadIdx.x >> 4);
  CacheTile t;
  t.row = tile / (uint32_t)A.heads;
  t.head = (int32_t)(tile - (uint32_t)t.row * (uint32_t)A.heads);
  t.at = -1;
  if (tile >= A.tiles) {
    t.row = -1;
    return t;
  }
  const int64_t slot = A.slots[t.row];
  if (slot >= 0 && slot < S.slots) {
    const uint32_t blk = (uint32_t)slot / (uint32_t)A.block_tokens;
    const uint32_t off = (uint32_t)slot - blk * (uint32_t)A.block_tokens;
    t.at = ((int64_t)blk * A.heads + t.head) * A.block_tokens + off;
  } else if (slot >= 0 && first && t.head == 0 && (lane & 15) == 0) {
    report(S.stats, HQ_ERR_INVALID_ARG);
  }
  return t;
}

template <int FMT>
__global__ __launch_bounds__(256) void hq_cache_write_kernel(hq_cache_io_args A) {
  const hq_cache_side& S = A.side[blockIdx.y];
  const int lane = threadIdx.x & 63;
  const CacheTile t = cache_tile(A, S, lane, true);
  const int c0 = (lane & 15) * 8;
  float v[8] = {};
  // every lane of a wave stays for the transform's lane moves
  if (t.at >= 0) {
    load8(S.x, t.row * S.ld + (int64_t)t.head * HQ_TILE + c0, A.x_bf16, v);
    const uint32_t dbits = sign_bits8(S.dmask, (int64_t)t.head * HQ_TILE + c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = flip(v[i], dbits, i);
  }
  const XSigns sg(lane);
  fwht128(v, sg);
  float am = amax_or_nan<8>(v);
  am = __builtin_elementwise_maximum(am, xor_lane_f<1>(am));
  am = __builtin_elementwise_maximum(am, xor_lane_f<2>(am));
  am = __builtin_elementwise_maximum(am, xor_lane_f<4>(am));
  am = __builtin_elementwise_maximum(am, xor_lane_f<8>(am));
  // a vector with an infinite or NaN value has no scale: codes 0, scale NaN
  const bool bad = !(am <= 3.4028234663852886e38f);
  if (bad) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    if (t.at >= 0 && (lane & 15) == 0 && S.stats) {
      atomicAdd(&S.stats->overflow_tiles, 1u);
      report(S.stats, HQ_ERR_OVERFLOW);
    }
  }
  if constexpr (FMT == kMx) {
    int32_t X;
    const uint32_t packed = mxfp4_x8(v, X);
    if (t.at < 0) return;
    *(uint32_t*)(S.codes + t.at * row_bytes<FMT>() + c0 / 2) = packed;
    if ((lane & 3) == 0) ((uint8_t*)S.scales)[t.at * 4 + ((lane & 15) >> 2)] = bad ? 0xFFu : (uint8_t)(X + 127);
  } else {
    const float top = FMT == kE4M3 ? 448.0f : 127.0f;
    // below 2^-100 the reciprocal could overflow: such a vector is stored as zeros
    const bool zero = bad || am < 0x1p-100f;
    const float inv = zero ? 0.0f : top / am;
    uint32_t packed[2] = {0u, 0u};
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      q[i] = v[i] * inv;
      if (FMT == kInt8) q[i] = __builtin_rintf(q[i]);
      q[i] = __builtin_fminf(__builtin_fmaxf(q[i], -top), top);
    }
    if constexpr (FMT == kE4M3) {
      packed[0] = e4m3x4(q[0], q[1], q[2], q[3]);
      packed[1] = e4m3x4(q[4], q[5], q[6], q[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) packed[i >> 2] |= ((uint32_t)(int32_t)q[i] & 0xFFu) << (8 * (i & 3));
    }
    if (t.at < 0) return;
    *(uint2*)(S.codes + t.at * row_bytes<FMT>() + c0) = make_uint2(packed[0], packed[1]);
    if ((lane & 15) == 0) ((float*)S.scales)[t.at] = bad ? __builtin_nanf("") : zero ? 0.0f : am / top;
  }
}

// The factor that an E8M0 byte stands for: 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float e8m0(uint32_t byte) {
  return byte == 255u ? __builtin_nanf("") : byte == 0u ? 0x1p-127f : __uint_as_float(byte << 23);
}

template <int FMT>
__global__ __launch_bounds__(256) void hq_cache_read_kernel(hq_cache_io_args A) {
  const hq_cache_side& S = A.side[0];
  const int lane = threadIdx.x & 63;
  const CacheTile t = cache_tile(A, S, lane, true);
  const int c0 = (lane & 15) * 8;
  float v[8] = {}, scale = 0.0f;
  if (t.at >= 0) {
    if constexpr (FMT == kMx) {
      const uint32_t w = *(const uint32_t*)(S.codes + t.at * row_bytes<FMT>() + c0 / 2);
      const float f = e8m0(((const uint8_t*)S.scales)[t.at * 4 + ((lane & 15) >> 2)]);
      scale = 1.0f;
      const v2f_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
      const v2f_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
      const v2f_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
      const v2f_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
      v[0] = a[0] * f; v[1] = a[1] * f; v[2] = b[0] * f; v[3] = b[1] * f;
      v[4] = c[0] * f; v[5] = c[1] * f; v[6] = d[0] * f; v[7] = d[1] * f;
    } else {
      const uint2 w = *(const uint2*)(S.codes + t.at * row_bytes<FMT>() + c0);
      scale = ((const float*)S.scales)[t.at];
      const uint32_t w2[2] = {w.x, w.y};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (FMT == kE4M3) {
          const v2f_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w2[h], false);
          const v2f_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w2[h], true);
          v[4 * h] = a[0]; v[4 * h + 1] = a[1]; v[4 * h + 2] = b[0]; v[4 * h + 3] = b[1];
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * h + i] = (float)(int8_t)(w2[h] >> (8 * i));
        }
      }
    }
  }
  const XSigns sg(lane);
  fwht128(v, sg);
  if (t.row < 0) return;
  // H of the codes first, then the scale: integer codes sum exactly
  const uint32_t dbits = sign_bits8(S.dmask, (int64_t)t.head * HQ_TILE + c0);
  const float f = scale * 0.0078125f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = t.at < 0 ? 0.0f : flip(v[i] * f, dbits, i);
  store8(A.y, t.row * A.ldy + (int64_t)t.head * HQ_TILE + c0, A.y_bf16, v);
}

// ----------------------------------------------------------------- attention
// One workgroup takes one KV head of one sequence and a run of its tokens (a
// split), each wave 32 tokens at a time.  Both products run on the matrix cores in
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

// What a wave loads for 32 tokens.
template <int FMT>
struct CacheStep {
  static constexpr int KW = FMT == kMx ? 4 : 8;  // words of 32 codes
  static constexpr int VW = FMT == kMx ? 1 : 2;  // words of 8 codes
  uint32_t k[2][KW];     // token 16 h + l % 16, dims 32 (l / 16) ..
  uint32_t v[2][4][VW];  // token 16 h + 4 (l / 16) + r, dims 8 (l % 16) ..
  float ks[2][4], vs[2][4];  // fp32 scales of those four tokens
  uint32_t kx[2], vx[2][4];  // MXFP4: the scale byte of k, the four bytes of v's tokens
  int32_t live[2];           // tokens of each half to attend to
};

struct CacheWalk {
  int32_t blk, off;  // block of the table and token inside it
  __device__ __forceinline__ void advance(int32_t by, int32_t bt) {
    off += by;
    while (off >= bt) {
      off -= bt;
      ++blk;
    }
  }
};

template <int FMT>
__device__ __forceinline__ void cache_load(const hq_cache_attn_args& A, const int32_t* table, int32_t head,
                                           CacheWalk w, int32_t t, int32_t end, int lane, CacheStep<FMT>& s) {
  const int n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int32_t live = end - t - 16 * h;
    live = live < 0 ? 0 : live > 16 ? 16 : live;
    int32_t b = 0;
    if (live > 0) {
      b = table[w.blk];
      if (b < 0 || b >= A.blocks) {
        live = 0;
        if (head == 0 && lane == 0) report(A.stats, HQ_ERR_INVALID_ARG);
      }
    }
    s.live[h] = live;
    if (live > 0) {
      const int64_t row = ((int64_t)b * A.heads_kv + head) * A.block_tokens + w.off;
      const uint8_t* kp = A.k_codes + (row + n) * row_bytes<FMT>() + g * (row_bytes<FMT>() / 4);
      const uint8_t* vp = A.v_codes + (row + 4 * g) * row_bytes<FMT>() + n * (row_bytes<FMT>() / 16);
#pragma unroll
      for (int i = 0; i < CacheStep<FMT>::KW; i += 4) {
        const uint4 x = *(const uint4*)(kp + 4 * i);
        s.k[h][i] = x.x; s.k[h][i + 1] = x.y; s.k[h][i + 2] = x.z; s.k[h][i + 3] = x.w;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (FMT == kMx) {
          s.v[h][r][0] = *(const uint32_t*)(vp + r * row_bytes<FMT>());
        } else {
          const uint2 x = *(const uint2*)(vp + r * row_bytes<FMT>());
          s.v[h][r][0] = x.x; s.v[h][r][1] = x.y;
        }
      }
      if constexpr (FMT == kMx) {
        s.kx[h] = ((const uint8_t*)A.k_scales)[(row + n) * 4 + g];
        const uint4 x = *(const uint4*)((const uint8_t*)A.v_scales + (row + 4 * g) * 4);
        s.vx[h][0] = x.x; s.vx[h][1] = x.y; s.vx[h][2] = x.z; s.vx[h][3] = x.w;
      } else {
        const float4 x = *(const float4*)((const float*)A.k_scales + row + 4 * g);
        const float4 y = *(const float4*)((const float*)A.v_scales + row + 4 * g);
        s.ks[h][0] = x.x; s.ks[h][1] = x.y; s.ks[h][2] = x.z; s.ks[h][3] = x.w;
        s.vs[h][0] = y.x; s.vs[h][1] = y.y; s.vs[h][2] = y.z; s.vs[h][3] = y.w;
      }
    }
    w.advance(16, A.block_tokens);
  }
}

constexpr int kQPitch = HQ_TILE + 8;  // bf16 of a query row in LDS
constexpr int kOPitch = HQ_TILE + 4;  // floats of an output row in LDS

template <int FMT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void hq_cache_attn_kernel(
    hq_cache_attn_args A) {
  __shared__ __attribute__((aligned(16))) float s_o[HQ_WAVES_PER_WG][16][kOPitch];
  __shared__ float s_m[HQ_WAVES_PER_WG][16], s_l[HQ_WAVES_PER_WG][16];
  uint16_t* s_q = (uint16_t*)&s_o[0][0][0];  // the query's terms, before the sums
  static_assert(3 * 16 * kQPitch * sizeof(uint16_t) <= sizeof(s_o), "the query fits the sums' place");
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = (int)readfirst((uint32_t)(tid >> 6));
  const uint32_t bh = blockIdx.x / (uint32_t)A.splits;
  const int32_t split = (int32_t)(blockIdx.x - bh * (uint32_t)A.splits);
  const int64_t b = bh / (uint32_t)A.heads_kv;
  const int32_t head = (int32_t)(bh - (uint32_t)b * (uint32_t)A.heads_kv);
  const int32_t G = A.group;
  const int64_t cap = (int64_t)A.max_blocks * A.block_tokens;
  int64_t len64 = A.seq_lens[b];
  if (len64 < 0 || len64 > cap) {
    if (split == 0 && head == 0 && tid == 0) report(A.stats, HQ_ERR_INVALID_ARG);
    len64 = len64 < 0 ? 0 : cap;
  }
  const int32_t len = (int32_t)len64;
  // the sequence's own tokens are shared out evenly, 128 (32 a wave) at least
  int32_t chunk = (int32_t)(((len64 + A.splits - 1) / A.splits + 127) & ~(int64_t)127);
  const int64_t begin64 = (int64_t)split * chunk;
  const int64_t pair0 = b * A.heads_q + (int64_t)head * G;
  if (begin64 >= len) {  // nothing here; the first split of an empty sequence still answers
    if (A.splits > 1) return;  // the join knows how many splits a length has
    const int grp = tid >> 4;
    const float z[8] = {};
    if (grp < G) store8(A.out, (pair0 + grp) * HQ_TILE + n * 8, A.out_bf16, z);
    return;
  }
  // ---- the query into the cache's coordinates, as three bf16 terms
  {
    const int grp = tid >> 4, c0 = n * 8;
    float v[8] = {};
    if (grp < G) {
      load8(A.q, (pair0 + grp) * HQ_TILE + c0, A.q_bf16, v);
      const uint32_t dbits = sign_bits8(A.k_dmask, (int64_t)head * HQ_TILE + c0);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = flip(v[i], dbits, i);
    }
    const XSigns sg(lane);
    fwht128(v, sg);
    uint32_t t[8][3];
#pragma unroll
    for (int i = 0; i < 8; ++i) three_terms(v[i] * A.qscale, t[i]);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint4 o;
      o.x = high_pair(t[0][i], t[1][i]);
      o.y = high_pair(t[2][i], t[3][i]);
      o.z = high_pair(t[4][i], t[5][i]);
      o.w = high_pair(t[6][i], t[7][i]);
      *(uint4*)(s_q + (i * 16 + grp) * kQPitch + c0) = o;
    }
  }
  __syncthreads();
  // step s of the contraction takes dims 32 (l / 16) + 8 s + j in lane l (the codes
  // that the lane's one run of 32 holds)
  uint32_t q[3][4][4];
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 x = *(const uint4*)(s_q + (i * 16 + n) * kQPitch + 32 * g + 8 * s);
      q[i][s][0] = x.x; q[i][s][1] = x.y; q[i][s][2] = x.z; q[i][s][3] = x.w;
    }
  __syncthreads();  // s_o takes the query's place

  v4_t acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
  float m = -__builtin_inff(), l = 0.0f;
  const int32_t per = chunk / HQ_WAVES_PER_WG;
  const int32_t begin = (int32_t)begin64 + wave * per;
  const int32_t end = min(len, begin + per);
  const int32_t* table = A.table + b * A.max_blocks;
  CacheWalk w;
  w.blk = begin / A.block_tokens;
  w.off = begin - w.blk * A.block_tokens;
  CacheStep<FMT> cur;
  if (begin < end) cache_load<FMT>(A, table, head, w, begin, end, lane, cur);
  for (int32_t t = begin; t < end; t += 32) {
    CacheStep<FMT> nxt;
    w.advance(32, A.block_tokens);
    if (t + 32 < end) cache_load<FMT>(A, table, head, w, t + 32, end, lane, nxt);
    if (cur.live[0] + cur.live[1] < 32) {
      // stale or absent tokens: their value codes count as zeros (their weight is
      // zero, but a stale code or scale may be a NaN)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * g + r >= cur.live[h]) {
#pragma unroll
            for (int i = 0; i < CacheStep<FMT>::VW; ++i) cur.v[h][r][i] = 0u;
            cur.ks[h][r] = cur.vs[h][r] = 0.0f;
            cur.vx[h][r] = 0x7F7F7F7Fu;
          }
    }
    float p[2][4];
    float top = -__builtin_inff();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float f = FMT == kMx ? e8m0(cur.kx[h]) : 1.0f;
      v4_t c = (v4_t){0.0f, 0.0f, 0.0f, 0.0f};
      uint32_t a[4][4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if constexpr (FMT == kMx) {
          pairs_of<FMT>(cur.k[h][s], f, a[s]);
        } else {
          pairs_of<FMT>(cur.k[h][2 * s], f, a[s]);
          pairs_of<FMT>(cur.k[h][2 * s + 1], f, a[s] + 2);
        }
      }
#pragma unroll
      for (int i = 2; i >= 0; --i)  // the small terms first
#pragma unroll
        for (int s = 0; s < 4; ++s) c = mfma_bf16(a[s], q[i][s], c);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = FMT == kMx ? c[r] : c[r] * cur.ks[h][r];
        if (4 * g + r >= cur.live[h]) x = -__builtin_inff();
        p[h][r] = x;
        top = __builtin_fmaxf(top, x);
      }
    }
    top = __builtin_fmaxf(top, swz_xor16(top));
    top = __builtin_fmaxf(top, lane_xor32(top));
    const float mn = __builtin_fmaxf(m, top);
    const float ref = mn == -__builtin_inff() ? 0.0f : mn;  // nothing seen yet
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] *= alpha;
    uint32_t pt[3][4];  // the weights' terms: k index 4 h + r
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t tt[4][3];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(p[h][r] - ref);
        l += e;
        three_terms(FMT == kMx ? e : e * cur.vs[h][r], tt[r]);
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        pt[i][2 * h] = high_pair(tt[0][i], tt[1][i]);
        pt[i][2 * h + 1] = high_pair(tt[2][i], tt[3][i]);
      }
    }
    // value codes: per token four words of two dims each, then per dim the tokens' pairs
    uint32_t vf[8][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        uint32_t x[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if constexpr (FMT == kMx) {
            pairs_of<FMT>(cur.v[h][r + e][0], e8m0((cur.vx[h][r + e] >> (8 * (n >> 2))) & 0xFFu), x[e]);
          } else {
            pairs_of<FMT>(cur.v[h][r + e][0], 1.0f, x[e]);
            pairs_of<FMT>(cur.v[h][r + e][1], 1.0f, x[e] + 2);
          }
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          vf[2 * d][2 * h + r / 2] = __builtin_amdgcn_perm(x[1][d], x[0][d], 0x05040100u);
          vf[2 * d + 1][2 * h + r / 2] = high_pair(x[0][d], x[1][d]);
        }
      }
#pragma unroll
    for (int i = 2; i >= 0; --i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = mfma_bf16(vf[j], pt[i], acc[j]);
    cur = nxt;
  }
  l += swz_xor16(l);
  l += lane_xor32(l);
  // acc[j][r] is dim 8 (4 g + r) + j of head n
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float* o = &s_o[wave][n][(4 * g + r) * 8];
    *(float4*)o = make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
    *(float4*)(o + 4) = make_float4(acc[4][r], acc[5][r], acc[6][r], acc[7][r]);
  }
  if (g == 0) {
    s_m[wave][n] = m;
    s_l[wave][n] = l;
  }
  __syncthreads();
  // ---- the four waves' sums under one maximum, one head per 16 lanes
  const int grp = tid >> 4, c0 = n * 8;
  float M = s_m[0][grp], L = 0.0f, v[8] = {};
#pragma unroll
  for (int x = 1; x < HQ_WAVES_PER_WG; ++x) M = __builtin_fmaxf(M, s_m[x][grp]);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
#pragma unroll
  for (int x = 0; x < HQ_WAVES_PER_WG; ++x) {
    const float f = __builtin_amdgcn_exp2f(s_m[x][grp] - ref);
    L = __builtin_fmaf(f, s_l[x][grp], L);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(f, s_o[x][grp][c0 + i], v[i]);
  }
  if (A.splits > 1) {
    if (grp >= G) return;
    const int64_t part = (pair0 + grp) * A.splits + split;
    store8(A.part_acc, part * HQ_TILE + c0, false, v);
    if (n == 0) {
      A.part_m[part] = M;
      A.part_l[part] = L;
    }
    return;
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / (L * 128.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
  const XSigns sg(lane);
  fwht128(v, sg);
  if (grp >= G) return;
  const uint32_t dbits = sign_bits8(A.v_dmask, (int64_t)head * HQ_TILE + c0);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = flip(v[i], dbits, i);
  store8(A.out, (pair0 + grp) * HQ_TILE + c0, A.out_bf16, v);
}

// Joins a query head's splits under one maximum, in order, and moves the result
// back: one workgroup per query head, 16 lanes per split.
__global__ __launch_bounds__(256) void hq_cache_join_kernel(hq_cache_attn_args A) {
  __shared__ float s_red[16];
  __shared__ float4 s_acc[16][32];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, grp = tid >> 4, c0 = n * 8;
  const int64_t pair = blockIdx.x;
  const int64_t b = pair / A.heads_q;
  const int32_t head = (int32_t)(pair - b * A.heads_q) / A.group;
  const int64_t cap = (int64_t)A.max_blocks * A.block_tokens;
  int64_t len = A.seq_lens[b];
  len = len < 0 ? 0 : len > cap ? cap : len;
  const int64_t chunk = ((len + A.splits - 1) / A.splits + 127) & ~(int64_t)127;
  const int32_t live = len > 0 ? (int32_t)((len + chunk - 1) / chunk) : 0;
  const float* pm = A.part_m + pair * A.splits;
  const float* pl = A.part_l + pair * A.splits;
  float M = -__builtin_inff();
  for (int32_t x = grp; x < live; x += 16) M = __builtin_fmaxf(M, pm[x]);
  if (n == 0) s_red[grp] = M;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 16; ++k) M = __builtin_fmaxf(M, s_red[k]);
  const float ref = M == -__builtin_inff() ? 0.0f : M;
  float L = 0.0f, v[8] = {};
  for (int32_t x = grp; x < live; x += 16) {
    const float f = __builtin_amdgcn_exp2f(pm[x] - ref);
    L = __builtin_fmaf(f, pl[x], L);
    float a[8];
    load8(A.part_acc, (pair * A.splits + x) * HQ_TILE + c0, false, a);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(f, a[i], v[i]);
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
    const float4 a0 = s_acc[k][2 * n], a1 = s_acc[k][2 * n + 1];
    v[0] += a0.x; v[1] += a0.y; v[2] += a0.z; v[3] += a0.w;
    v[4] += a1.x; v[5] += a1.y; v[6] += a1.z; v[7] += a1.w;
    L += s_red[k];
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / (L * 128.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
  const XSigns sg(lane);
  fwht128(v, sg);
  const uint32_t dbits = sign_bits8(A.v_dmask, (int64_t)head * HQ_TILE + c0);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = flip(v[i], dbits, i);
  store8(A.out, pair * HQ_TILE + c0, A.out_bf16, v);
}

}  // namespace

#define HQ_CACHE_FORMATS(KERNEL, FMT, GRID, STREAM, ARGS)                                        \
  switch (FMT) {                                                                                 \
    case HQ_INT8: hipLaunchKernelGGL(KERNEL<kInt8>, GRID, dim3(256), 0, STREAM, ARGS); break;    \
    case HQ_E4M3: hipLaunchKernelGGL(KERNEL<kE4M3>, GRID, dim3(256), 0, STREAM, ARGS); break;    \
    default: hipLaunchKernelGGL(KERNEL<kMx>, GRID, dim3(256), 0, STREAM, ARGS);                  \
  }

int hq_launch_cache_write(const hq_cache_io_args& a, int format, int sides, void* stream) {
  const dim3 grid((a.tiles + 15) / 16, (uint32_t)sides);
  HQ_CACHE_FORMATS(hq_cache_write_kernel, format, grid, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

int hq_launch_cache_read(const hq_cache_io_args& a, int format, void* stream) {
  const dim3 grid((a.tiles + 15) / 16);
  HQ_CACHE_FORMATS(hq_cache_read_kernel, format, grid, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

int hq_launch_cache_attention(const hq_cache_attn_args& a, int format, void* stream) {
  const dim3 grid((uint32_t)(a.batch * a.heads_kv * a.splits));
  HQ_CACHE_FORMATS(hq_cache_attn_kernel, format, grid, (hipStream_t)stream, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(hq_cache_join_kernel, dim3((uint32_t)(a.batch * a.heads_q)), dim3(256), 0,
                       (hipStream_t)stream, a);
  return (int)hipGetLastError();
}
