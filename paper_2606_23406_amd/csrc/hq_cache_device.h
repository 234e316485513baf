// What the kernels over the fixed-rate key-value cache share: head vectors in and out of
// registers, the chunks of a call's sequences, and a wave's way over a sequence's tokens.
#ifndef HQ_CACHE_DEVICE_H
#define HQ_CACHE_DEVICE_H
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

// Casts a vector of 16 lanes' transformed values, sigma times y (TwSigns), and stores it as
// vector vec of the cache where it is live.
template <int FMT>
__device__ __forceinline__ void cache_put(const hq_cache_side& S, float* v, bool live, int64_t vec, int lane,
                                          const TwSigns& sg) {
  const int c0 = (lane & 15) * 8;
  float am = amax_or_nan<8>(v);
  am = __builtin_elementwise_maximum(am, dpp_xor<1>(am));
  am = __builtin_elementwise_maximum(am, dpp_xor<2>(am));
  am = __builtin_elementwise_maximum(am, swz_xor4(am));
  am = __builtin_elementwise_maximum(am, dpp_xor<8>(am));
  // a vector with an infinite or NaN value has no scale: codes 0, scale NaN
  const bool bad = !(am <= 3.4028234663852886e38f);
  if (__builtin_expect(bad, 0)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (live && (lane & 15) == 0 && S.stats) {
      atomicAdd(&S.stats->overflow_tiles, 1u);
      report(S.stats, HQ_ERR_OVERFLOW);
    }
  }
  if constexpr (FMT == kMx) {
    int32_t X;
    const uint32_t packed = mxfp4_x8(v, X) ^ (sg.sigma ? 0x88888888u : 0u);
    if (!live) return;
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
      packed.x = e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      packed.y = e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    } else {
      packed = int8x8(v, inv);
    }
    if (!live) return;
    *(uint2*)(S.codes + vec * row_bytes<FMT>() + c0) = packed;
    if ((lane & 15) == 0) ((float*)S.scales)[vec] = bad ? __builtin_nanf("") : zero ? 0.0f : over(am, top);
  }
}

typedef float v4_t __attribute__((ext_vector_type(4)));
typedef __bf16 v8b_t __attribute__((ext_vector_type(8)));
typedef uint32_t v4w_t __attribute__((ext_vector_type(4)));

// The high halves of two words: two bf16 from two fp32 by truncation, lo first.
__device__ __forceinline__ uint32_t high_pair(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
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
__device__ __forceinline__ int32_t cache_len(const hq_cache_attn_args& A, int64_t b, bool tell) {
  const int64_t cap = (int64_t)A.max_blocks * A.block_tokens;
  const int64_t len = A.seq_lens[b];
  if (len >= 0 && len <= cap) return (int32_t)len;
  if (tell) report(A.stats, HQ_ERR_INVALID_ARG);
  return len < 0 ? 0 : (int32_t)cap;
}

// Which tokens of a sequence an attention looks at: all of them; those of a window with the
// first ones (sinks); those before and of a tree of drafted tokens, the sequence's last ones.
constexpr int kAll = 0, kWindow = 1, kTree = 2;

// Tokens [0, sinks) and [low, len).  The way over them goes by groups of 16, with `gap` tokens
// between the sinks' last group and the window's first left out: token i on the way is token
// i below the sinks' end (rounded up), i + gap behind it.
struct CacheSpan {
  int32_t len;         // 0: nothing
  int32_t low, sinks;  // sinks <= low
  int32_t rows, from;  // drafted tokens, and the first one's row
  __device__ __forceinline__ int32_t turn() const { return (sinks + 15) & ~15; }
  __device__ __forceinline__ int32_t gap() const { return max((low & ~15) - turn(), 0); }
  __device__ __forceinline__ int32_t seen() const { return len - gap(); }
  // bit i: token at + i is looked at
  __device__ __forceinline__ uint32_t bits(int32_t at) const {
    auto below = [&](int32_t t) { return (1u << min(max(t - at, 0), 16)) - 1u; };
    return below(sinks) | (below(len) & ~below(low));
  }
};

template <int MODE>
__device__ __forceinline__ CacheSpan cache_span(const hq_cache_attn_args& A, int32_t len, int32_t rows, int32_t from) {
  CacheSpan s = {len, 0, 0, rows, from};
  if (MODE != kAll && A.window) {
    s.low = max(len - rows - A.window, 0);
    s.sinks = min(A.sinks, s.low);
  }
  return s;
}

// Drafted tokens of sequence b (0 for the other modes).  Places that are out of order or range,
// more tokens than the call's bound or than the sequence: reported, and none.
template <int MODE>
__device__ __forceinline__ int32_t cache_rows(const hq_cache_attn_args& A, int64_t b, int32_t len, bool tell,
                                              int32_t& from) {
  from = 0;
  if (MODE != kTree) return 0;
  from = A.starts[b];
  const int32_t to = A.starts[b + 1];
  const bool ok = from >= 0 && to >= from && to <= A.rows && to - from <= A.max_rows && to - from <= len;
  if (!ok && tell) report(A.stats, HQ_ERR_INVALID_ARG);
  return ok ? to - from : 0;
}

template <int MODE>
__device__ __forceinline__ CacheSpan cache_span_of(const hq_cache_attn_args& A, int64_t b, bool tell) {
  int32_t from;
  const int32_t len = cache_len(A, b, tell), rows = cache_rows<MODE>(A, b, len, tell, from);
  return cache_span<MODE>(A, MODE == kTree && rows == 0 ? 0 : len, rows, from);
}

struct CacheItem {
  int32_t b;       // -1: behind the last item
  int32_t n;       // chunks of this sequence (an empty one has one, which writes its zeros)
  int32_t first;   // the sequence's first item
  int32_t at;      // which of its chunks
  int32_t tile;    // which of a tree's row tiles
  int32_t chunk;
  CacheSpan span;  // its tokens
};

// Row tiles of a sequence's tree, each with all its chunks; one for the other modes and for
// none.
template <int MODE>
__device__ __forceinline__ int32_t cache_tiles(const hq_cache_attn_args& A, int32_t rows) {
  if (MODE != kTree) return 1;
  return max((rows * A.group + (1 << A.tile_shift) - 1) >> A.tile_shift, 1);
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
// `total`: all tokens, once for each row tile; `mine`: a lane's or thread's own sequence's, -1
// without one, and its row tiles; `sum` adds a number over all of these.
template <typename SUM>
__device__ __forceinline__ uint32_t cache_chunk(const hq_cache_attn_args& A, int64_t total, int32_t mine, int32_t tiles,
                                                SUM sum) {
  const int64_t even = (total * A.heads_kv + HQ_CACHE_WG_TARGET - 1) / HQ_CACHE_WG_TARGET;
  const int64_t few = (HQ_CACHE_WG_TARGET + HQ_CACHE_WG_TARGET / 32) / (uint32_t)A.heads_kv;
  uint32_t chunk = HQ_CACHE_LEAST;
  for (int e = 8; e <= 16; ++e) {
    const int64_t c = min(((even * e >> 3) + kStep - 1) & -(int64_t)kStep, (int64_t)1 << 30);
    chunk = max(chunk, readfirst((uint32_t)c));
    if (A.batch > few) break;
    // about: a length a hair over a multiple may count as the multiple
    const float per = __builtin_amdgcn_rcpf((float)chunk) * 0.999999f;
    if (sum(mine < 0 ? 0u : max(1u, (uint32_t)__builtin_ceilf((float)mine * per)) * (uint32_t)tiles) <= few) break;
  }
  return chunk;
}

// Whole steps of all waves, about as many in each of a sequence's n chunks.
__device__ __forceinline__ int32_t even_chunk(int32_t len, int32_t n) {
  return (len + n * kStep - 1) / (n * kStep) * kStep;
}

template <int MODE>
__device__ __forceinline__ CacheItem cache_item(const hq_cache_attn_args& A, int32_t j, int lane, bool tell) {
  CacheItem it;
  it.b = -1;
  if (!A.join) {  // one chunk each
    const int32_t b = MODE == kTree ? j / A.max_tiles : j;
    if (b >= A.batch) return it;
    it.b = b;
    it.first = j;
    it.n = 1;
    it.at = 0;
    it.tile = MODE == kTree ? j - b * A.max_tiles : 0;
    const CacheSpan s = cache_span_of<MODE>(A, it.b, true);
    it.span = {(int32_t)readfirst((uint32_t)s.len), (int32_t)readfirst((uint32_t)s.low),
               (int32_t)readfirst((uint32_t)s.sinks), (int32_t)readfirst((uint32_t)s.rows),
               (int32_t)readfirst((uint32_t)s.from)};
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
    if (MODE != kTree && j >= it.first + it.n) return it;
    it.b = (int32_t)readfirst((uint32_t)lo);
    const CacheSpan s = cache_span_of<MODE>(A, it.b, false);
    it.span = {(int32_t)readfirst((uint32_t)s.len), (int32_t)readfirst((uint32_t)s.low),
               (int32_t)readfirst((uint32_t)s.sinks), (int32_t)readfirst((uint32_t)s.rows),
               (int32_t)readfirst((uint32_t)s.from)};
  } else {
    static_assert(HQ_CACHE_UNPLANNED <= 64, "");
    const bool in = lane < A.batch;
    const CacheSpan s = in ? cache_span_of<MODE>(A, lane, tell) : CacheSpan{-1, 0, 0, 0, 0};
    const int32_t len = MODE == kAll ? s.len : s.seen();
    const int32_t tiles = cache_tiles<MODE>(A, s.rows);
    const uint64_t of = (uint64_t)max(len, 0) * (uint32_t)tiles;  // below 2^37
    uint32_t sum0 = (uint32_t)of & 0xFFFFu, sum1 = (uint32_t)(of >> 16);
    wave_scan_incl2(sum0, sum1);
    const int64_t total =
        ((int64_t)__builtin_amdgcn_readlane(sum1, 63) << 16) + (uint32_t)__builtin_amdgcn_readlane(sum0, 63);
    const uint32_t chunk = cache_chunk(A, total, len, tiles, [](uint32_t n) { return wave_total(n); });
    const uint32_t n = in ? cache_parts(len, chunk) : 0u;
    const int32_t incl = (int32_t)wave_scan_incl(n * (uint32_t)tiles);
    if (j >= __builtin_amdgcn_readlane(incl, 63)) return it;
    const int at = __popcll(__ballot(incl <= j));
    it.b = at;
    it.n = (int32_t)__builtin_amdgcn_readlane(n, at);
    it.first = __builtin_amdgcn_readlane(incl, at) - it.n * (int32_t)__builtin_amdgcn_readlane(tiles, at);
    it.span = cache_span<MODE>(A, __builtin_amdgcn_readlane(s.len, at),
                               MODE == kTree ? __builtin_amdgcn_readlane(s.rows, at) : 0,
                               MODE == kTree ? __builtin_amdgcn_readlane(s.from, at) : 0);
  }
  if (MODE == kTree) {
    const int32_t tiles = cache_tiles<MODE>(A, it.span.rows);
    it.at = (j - it.first) / tiles;
    it.tile = j - it.first - it.at * tiles;
    if (it.at >= it.n) it.b = -1;  // behind the last sequence's
  } else {
    it.at = j - it.first;
    it.tile = 0;
  }
  it.chunk = even_chunk(MODE == kAll ? it.span.len : it.span.seen(), it.n);
  return it;
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

// Where a wave stands in its sequence, all of whose tokens it goes through: token off of block blk
// of the table row, and that block's head as buffers.  The ids of 64 blocks ahead are one per
// lane, so that following the table costs a lane read and not a load that the next loads'
// addresses wait for.
struct CacheWalk {
  // What a fetch returns of its two halves: tokens of each to attend to.
  struct Look {
    int32_t live[2];
  };
  const int32_t* table;
  int32_t last;  // the sequence's last block
  int32_t head, blk, off;
  int32_t first, ids;  // lane l: block first + l
  __amdgpu_buffer_rsrc_t k, v, ks, vs;
  bool bad;  // the block lies outside the cache: its buffers are empty
  // To token `begin`.
  __device__ __forceinline__ void start(const hq_cache_attn_args& A, const CacheItem& it, int32_t of, int32_t begin) {
    table = A.table + (int64_t)it.b * A.max_blocks;
    head = of;
    last = (it.span.len - 1) / A.block_tokens;
    blk = min(begin / A.block_tokens, last);
    off = begin - blk * A.block_tokens;
  }
  __device__ __forceinline__ void ask(const hq_cache_attn_args&, int32_t, int lane) { ask(lane); }
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
  // past them.
  template <int FMT>
  __device__ __forceinline__ Look fetch(const hq_cache_attn_args& A, int32_t t, int32_t end, int lane, uint8_t* step) {
    using R = CacheRing<FMT>;
    constexpr uint32_t RPL = 1024 / R::RB, CPR = R::RB / 16;  // rows of a load, chunks of a row
    const uint32_t row_in = lane / CPR, chunk = lane % CPR;
    const uint32_t from = row_in * R::RB + (chunk ^ R::swizzle(row_in)) * 16;
    Look look;
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
      look.live[h] = bad ? 0 : min(max(end - t - 16 * h, 0), 16);
      const uint32_t place = look.live[h] ? off : 0;
      off += 16;
      uint8_t* to = step + h * R::HALF;
#pragma unroll
      for (uint32_t i = 0; i < 16 / RPL; ++i) {
        const uint32_t rows = place * R::RB + i * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(k, (lds_void*)(to + i * 1024), 16, from, rows, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(v, (lds_void*)(to + R::V + i * 1024), 16, from, rows, 0, 0);
      }
      const uint32_t token = (lane & 15) * 4;  // four times over
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ks, (lds_void*)(to + R::SCALES), 4, token, place * 4, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vs, (lds_void*)(to + R::SCALES + 256), 4, token, place * 4, 0, 0);
    }
    return look;
  }
  __device__ __forceinline__ bool cut(const Look& x) const { return x.live[0] + x.live[1] < 32; }
  __device__ __forceinline__ bool dead(const Look& x, int32_t, int h, int32_t i) const { return i >= x.live[h]; }
};

// A scalar base for lane offsets: addresses per lane would live through the whole loop.
__device__ __forceinline__ const uint8_t* uniform(const void* p, int64_t bytes) {
  const uint64_t a = (uint64_t)p + bytes;
  return (const uint8_t*)((uint64_t)readfirst((uint32_t)(a >> 32)) << 32 | readfirst((uint32_t)a));
}
typedef __attribute__((address_space(1))) const void glb_void;

// The same of a window or a tree, some of whose tokens are left out.  A half's place is formed
// from its token by a multiplication, with no state from half to half but the block ids.  Every
// instruction counts, scalar ones too (a wave issues one in some 7 cycles): what a step's
// masks go by is formed when one is needed.  (Windows of 300 tokens 9.1 us, 9.5 with buffers of a
// block and a window's state; whole sequences are bound by memory and take 1 to 3 % longer so.)
struct SpanWalk {
  using Look = uint32_t;  // what a fetch returns
  const int32_t* table;
  CacheSpan span;
  int32_t gap, jump, head, last;  // last: the sequence's last block
  int32_t ctx, open, sinks;       // all rows see [0, sinks) and [open, ctx)
  int32_t first, ids;
  int64_t stride, offset;         // vectors of a block, those before the head's
  __device__ __forceinline__ void start(const hq_cache_attn_args& A, const CacheItem& it, int32_t of, int32_t) {
    table = A.table + (int64_t)it.b * A.max_blocks;
    span = it.span;
    gap = span.gap();
    jump = gap ? span.turn() : 0x7FFFFFFF;
    head = of;
    last = (span.len - 1) / A.block_tokens;
    ctx = span.len - span.rows;
    open = A.window ? ctx + span.rows - A.window : 0;
    sinks = A.sinks;
    stride = (int64_t)A.heads_kv * A.block_tokens;
    offset = (int64_t)of * A.block_tokens;
  }
  __device__ __forceinline__ int32_t real(int32_t t) const { return t < jump ? t : t + gap; }
  __device__ __forceinline__ int32_t block(const hq_cache_attn_args& A, int32_t at) const {
    return min((int32_t)A.by_block.of((uint32_t)at), last);
  }
  __device__ __forceinline__ void ask(const hq_cache_attn_args& A, int32_t begin, int lane) {
    ask(block(A, real(begin)), lane);
  }
  __device__ __forceinline__ void ask(int32_t blk, int lane) {
    first = blk;
    ids = table[min(blk + lane, last)];
  }
  __device__ __forceinline__ void got() { asm volatile("" : "+v"(ids)); }
  template <int FMT, bool>
  __device__ __forceinline__ void enter(const hq_cache_attn_args&, int) {}
  // Starts the loads of the 32 tokens from t on into `step`.  Returns 1 + 2 + 4 where all rows see
  // all of them, else 2 and 4 for the halves with tokens at all; one without loads the cache's
  // first ones.
  template <int FMT>
  __device__ __forceinline__ Look fetch(const hq_cache_attn_args& A, int32_t t, int32_t end, int lane, uint8_t* step) {
    using R = CacheRing<FMT>;
    constexpr uint32_t RPL = 1024 / R::RB, CPR = R::RB / 16;  // rows of a load, chunks of a row
    const uint32_t row_in = lane / CPR, chunk = lane % CPR;
    const uint32_t from = row_in * R::RB + (chunk ^ R::swizzle(row_in)) * 16, token = (lane & 15) * 4;
    uint32_t all = 1, some = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t at = real(t + 16 * h), blk = block(A, at);
      if (blk - first >= 64) {
        ask(blk, lane);
        got();
      }
      const int32_t id = __builtin_amdgcn_readlane(ids, blk - first);
      const bool in = t + 16 * h < end, ok = in && (uint32_t)id < (uint32_t)A.blocks;
      if (in && !ok && head == 0 && lane == 0) report(A.stats, HQ_ERR_INVALID_ARG);
      if (!ok || at + 16 > ctx || (at < open && at + 16 > sinks)) all = 0;
      if (ok) some |= 2u << h;
      const int64_t row = ok ? id * stride + offset + (at - blk * A.block_tokens) : 0;
      uint8_t* to = step + h * R::HALF;
      const uint8_t *k = uniform(A.k_codes, row * R::RB), *v = uniform(A.v_codes, row * R::RB);
      glb_void *const kl = (glb_void*)(k + from), *const vl = (glb_void*)(v + from);
      __builtin_amdgcn_global_load_lds(kl, (lds_void*)to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(vl, (lds_void*)(to + R::V), 16, 0, 0);
      if constexpr (RPL < 16) {  // the offset moves both places
        __builtin_amdgcn_global_load_lds(kl, (lds_void*)to, 16, 1024, 0);
        __builtin_amdgcn_global_load_lds(vl, (lds_void*)(to + R::V), 16, 1024, 0);
      }
      const uint8_t *ks = uniform(A.k_scales, row * 4), *vs = uniform(A.v_scales, row * 4);
      __builtin_amdgcn_global_load_lds((glb_void*)(ks + token), (lds_void*)(to + R::SCALES), 4, 0, 0);
      __builtin_amdgcn_global_load_lds((glb_void*)(vs + token), (lds_void*)(to + R::SCALES + 256), 4, 0, 0);
    }
    return all | some;
  }
  __device__ __forceinline__ bool cut(Look seen) const { return !(seen & 1); }
  __device__ __forceinline__ bool dead(Look seen, int32_t t, int h, int32_t i) const {
    return !((seen >> h) & 2) || !((span.bits(real(t + 16 * h)) >> i) & 1);
  }
  // Of the 32 tokens from t on: each half's first and the bits of those that anybody sees.
  __device__ __forceinline__ void about(int32_t t, uint32_t seen, int32_t (&live)[2], int32_t (&at)[2]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      at[h] = real(t + 16 * h);
      live[h] = (seen >> h) & 2 ? (int32_t)span.bits(at[h]) : 0;
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

constexpr int kQPitch = HQ_TILE + 8;  // bf16 of a query row in LDS
constexpr int kOPitch = HQ_TILE + 4;  // floats of an output row in LDS

// v * 1 / (128 sum) moved back to the head's own coordinates.
__device__ __forceinline__ void cache_finish(const hq_cache_attn_args& A, float L, float* v, int32_t head, int lane) {
  const float inv = L == 0.0f ? 0.0f : 1.0f / (L * 128.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
  const TwSigns sg(lane);
  fwht128_tw(v, sg);
  uint4 d = sign_words(A.v_dsign16, head * HQ_TILE + (lane & 15) * 8);
  const uint32_t sigma = sg.sigma | sg.sigma >> 16;
  d.x ^= sigma; d.y ^= sigma; d.z ^= sigma; d.w ^= sigma;
  flip8(v, d);
}

}  // namespace

#endif
