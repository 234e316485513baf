// gfx950 kernels of rotary positions: the table of cosines and sines
// (hq_rope_table), rows turned by it (hq_rope), and new keys and values cast into
// their cache's slots with the keys turned on the way (hq_cache_append).
//
// Pair i of a head, (a, b), is turned by the angle of its row's position on the
// pair's axis: (a c - b s, b c + a s), c and s from the table; transposed, which is
// the gradient, with -s.  Each product and sum is one fp32 rounding.
//
// 16 lanes take a head vector, 8 values each.  Pairs (i, i + pairs) lie in two lanes
// pairs / 8 apart, which trade their values; pairs (2 i, 2 i + 1) in one lane.
#include <hip/hip_runtime.h>

#include "hq_cache_device.h"

#pragma clang fp contract(off)

namespace {

// A row's positions, one per axis.
struct Positions {
  int32_t p[4];
  bool ok;  // all of them are in the table
};

__device__ __forceinline__ Positions load_positions(const hq_turns& T, uint32_t row, int lane) {
  Positions x;
  x.ok = true;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    x.p[a] = a == 0 || a < T.axes ? T.pos[(int64_t)row * T.axes + a] : 0;
    x.ok &= (uint32_t)x.p[a] < (uint32_t)T.count;
  }
  // a row of padding is left alone without a word
  if (!x.ok && x.p[0] >= 0 && (lane & 15) == 0) report(T.stats, HQ_ERR_INVALID_ARG);
#pragma unroll
  for (int a = 0; a < 4; ++a) x.p[a] = x.ok ? x.p[a] : 0;
  return x;
}

__device__ __forceinline__ int32_t axis_position(const hq_turns& T, uint32_t pair, const int32_t (&p)[4]) {
  const uint32_t at = pair >> 4;
  const uint32_t w = at == 0 ? T.axis[0] : at == 1 ? T.axis[1] : at == 2 ? T.axis[2] : T.axis[3];
  const uint32_t a = (w >> (2 * (pair & 15u))) & 3u;
  return a == 0 ? p[0] : a == 1 ? p[1] : a == 2 ? p[2] : p[3];
}

// What one row's turn is to a lane: cosines and sines of its values' pairs (of
// interleaved pairs the first four), the sines with the sign that they enter with.
struct Turn {
  float c[8], s[8];
  bool in;  // the lane's values are among the turned ones
};

__device__ __forceinline__ Turn load_turn(const hq_turns& T, const int32_t (&p)[4], int lane, bool transposed) {
  Turn t;
  const uint32_t n = lane & 15, half = (uint32_t)T.pairs >> 3;  // lanes of a half
  t.in = n < 2 * half;
  const uint32_t lower = n < half, turn = transposed ? 0x80000000u : 0u;
  if (T.interleaved) {
    const uint32_t p0 = t.in ? 4 * n : 0u;
    if (T.runs) {
      const float* at = T.table + (int64_t)axis_position(T, p0, p) * 2 * T.pairs + p0;
      const float4 c = *(const float4*)at, s = *(const float4*)(at + T.pairs);
      t.c[0] = c.x; t.c[1] = c.y; t.c[2] = c.z; t.c[3] = c.w;
      t.s[0] = s.x; t.s[1] = s.y; t.s[2] = s.z; t.s[3] = s.w;
    } else {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const float* at = T.table + (int64_t)axis_position(T, p0 + j, p) * 2 * T.pairs + p0 + j;
        t.c[j] = at[0];
        t.s[j] = at[T.pairs];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) t.s[j] = xor_sign(t.s[j], turn);
  } else {
    const uint32_t p0 = lower ? 8 * n : t.in ? 8 * (n - half) : 0u;
    if (T.runs) {
      const float* at = T.table + (int64_t)axis_position(T, p0, p) * 2 * T.pairs + p0;
      load8(at, 0, false, t.c);
      load8(at, T.pairs, false, t.s);
    } else {
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) {
        const float* at = T.table + (int64_t)axis_position(T, p0 + j, p) * 2 * T.pairs + p0 + j;
        t.c[j] = at[0];
        t.s[j] = at[T.pairs];
      }
    }
    const uint32_t sign = turn ^ (lower ? 0x80000000u : 0u);
#pragma unroll
    for (int j = 0; j < 8; ++j) t.s[j] = xor_sign(t.s[j], sign);
  }
  return t;
}

// Every lane of a wave takes part.
__device__ __forceinline__ void apply_turn(const hq_turns& T, const Turn& t, int lane, float* v) {
  if (T.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = v[2 * j], b = v[2 * j + 1];
      v[2 * j] = t.in ? a * t.c[j] - b * t.s[j] : a;
      v[2 * j + 1] = t.in ? b * t.c[j] + a * t.s[j] : b;
    }
    return;
  }
  float o[8];
  if (T.pairs == 64) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = dpp_xor<8>(v[j]);
  } else {
    const int n = lane & 15, half = T.pairs >> 3;
    const int from = (lane & 48) | (n < half ? n + half : n < 2 * half ? n - half : n);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = __shfl(v[j], from, 64);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = t.in ? v[j] * t.c[j] + o[j] * t.s[j] : v[j];
}

// Bound by its 64-bit arithmetic (sine, cosine, a division): 131072 positions of 64 pairs, 67 MB, take
// 34.9 us, at a large copy's rate 13.1; 4096 of them 5.7, a launch and little else.
__global__ __launch_bounds__(256) void hq_rope_table_kernel(hq_rope_table_args A) {
  const int64_t n = A.count * A.pairs;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
    const int64_t p = x / A.pairs, i = x - p * A.pairs;
    double s, c;
    sincos((double)p * A.freqs[i], &s, &c);
    A.table[2 * p * A.pairs + i] = (float)(c * A.factor);
    A.table[(2 * p + 1) * A.pairs + i] = (float)(s * A.factor);
  }
}

// 8 values of an array whose type the launch goes by.
template <bool BF16>
struct Raw {
  uint4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    if constexpr (BF16) {
      w[0] = *(const uint4*)((const uint16_t*)p + i);
    } else {
      w[0] = *(const uint4*)((const float*)p + i);
      w[1] = *(const uint4*)((const float*)p + i + 4);
    }
  }
  __device__ __forceinline__ void expand(float* v) const {
    if constexpr (BF16) {
      expand8({w[0], w[0]}, true, v);
    } else {
      expand8({w[0], w[1]}, false, v);
    }
  }
};

typedef uint32_t v4q_t __attribute__((ext_vector_type(4)));

// store8, past the caches where `past`.
__device__ __forceinline__ void store8_past(void* p, int64_t i, bool bf16, bool past, const float* v) {
  if (!past) return store8(p, i, bf16, v);
  if (bf16) {
    const v4q_t o = {cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
    __builtin_nontemporal_store(o, (v4q_t*)((uint16_t*)p + i));
  } else {
    v4q_t o[2];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k >> 2][k & 3] = __float_as_uint(v[k]);
    __builtin_nontemporal_store(o[0], (v4q_t*)((float*)p + i));
    __builtin_nontemporal_store(o[1], (v4q_t*)((float*)p + i + 4));
  }
}

// A lane group takes up to H heads of a row, groups apart: the row's positions and table
// lines are loaded once for them, and neighbouring lane groups have neighbouring heads.
// Bound by memory: 7800 rows of 20 heads in bf16, 84 MB with the table's lines, take 15.5 us,
// at a large copy's rate 16.4 (some of the rows are in the last cache).  16 rows of 32 heads: a
// launch and one chain of two loads, position and then table, 4.6 us on the GPU.
template <int H, bool BF16>
__device__ __forceinline__ void rope_tile(const hq_rope_args& A, const hq_turns& T, uint32_t tile, bool in) {
  const int lane = threadIdx.x & 63, c0 = (lane & 15) * 8;
  const uint32_t row = A.by_groups.of(tile), head0 = tile - row * (uint32_t)A.groups;
  Raw<BF16> raw[H];
#pragma unroll
  for (uint32_t i = 0; i < H; ++i)
    raw[i].load(A.x, (int64_t)row * A.ldx + (min(head0 + i * (uint32_t)A.groups, (uint32_t)A.heads - 1) * HQ_TILE + c0));
  const Positions p = load_positions(T, row, lane);
  const Turn t = load_turn(T, p.p, lane, A.transposed);
#pragma unroll
  for (uint32_t i = 0; i < H; ++i) {
    const uint32_t head = head0 + i * (uint32_t)A.groups;
    float v[8];
    raw[i].expand(v);
    apply_turn(T, t, lane, v);
    if (in && p.ok && head < (uint32_t)A.heads)
      store8_past(A.y, (int64_t)row * A.ldy + (head * HQ_TILE + c0), A.y_bf16, A.past, v);
  }
}

template <int H, bool BF16>
__global__ __launch_bounds__(256) void hq_rope_kernel(hq_rope_args A) {
  const uint32_t t = blockIdx.x * 16u + (threadIdx.x >> 4);
  rope_tile<H, BF16>(A, A.turn, min(t, A.tiles - 1), t < A.tiles);
}

// Workgroups of the keys, of the values, of the queries.  A lane group takes U heads of a row
// (8192 rows of 8 heads and their 32 query heads in bf16 to E4M3: 42.2 us with four, 44.3 with
// two, 46.3 with one).  Bound by memory: 189 MB, which a large copy moves in 37 us; the queries
// are two thirds of it.
template <int FMT, bool BF16, int U>
__global__ __launch_bounds__(256) void hq_cache_append_kernel(hq_cache_append_args A) {
  const uint32_t at = blockIdx.x / A.side_groups;
  if (at >= (uint32_t)A.sides) {
    const uint32_t t = (blockIdx.x - (uint32_t)A.sides * A.side_groups) * 16u + (threadIdx.x >> 4);
    if (A.q.per == 4)
      rope_tile<4, BF16>(A.q, A.turn, min(t, A.q.tiles - 1), t < A.q.tiles);
    else
      rope_tile<1, BF16>(A.q, A.turn, min(t, A.q.tiles - 1), t < A.q.tiles);
    return;
  }
  const hq_cache_side& S = A.side[at];
  const int lane = threadIdx.x & 63, c0 = (lane & 15) * 8;
  const uint32_t t = (blockIdx.x - at * A.side_groups) * 16u + (threadIdx.x >> 4), tile = min(t, A.tiles - 1);
  const uint32_t row = A.by_groups.of(tile), head0 = tile - row * (uint32_t)A.groups;
  const int64_t slot = A.slots[row];
  Raw<BF16> raw[U];
  uint4 d[U];
#pragma unroll
  for (uint32_t i = 0; i < U; ++i) {
    const uint32_t col = min(head0 + i * (uint32_t)A.groups, (uint32_t)A.heads - 1) * HQ_TILE + c0;
    raw[i].load(S.x, (int64_t)row * S.ld + col);
    d[i] = sign_words(S.dsign16, col);
  }
  // a row without positions leaves both sides of its slot as they were
  const Positions p = load_positions(A.turn, row, lane);
  Turn turn;
  if (at == 0) turn = load_turn(A.turn, p.p, lane, false);
  const bool here = slot >= 0 && slot < S.slots;
  if (slot >= S.slots && head0 == 0 && (lane & 15) == 0) report(S.stats, HQ_ERR_INVALID_ARG);
  const uint32_t s = here ? (uint32_t)slot : 0u, blk = A.by_block.of(s);
  const int64_t vec0 = (int64_t)(blk * (uint64_t)(uint32_t)A.heads) * A.block_tokens + (s - blk * (uint32_t)A.block_tokens);
  const TwSigns sg(lane);
#pragma unroll
  for (uint32_t i = 0; i < U; ++i) {
    const uint32_t head = head0 + i * (uint32_t)A.groups;
    float v[8];
    raw[i].expand(v);
    if (at == 0) apply_turn(A.turn, turn, lane, v);
    flip8(v, d[i]);
    fwht128_tw(v, sg);
    cache_put<FMT>(S, v, here && p.ok && t < A.tiles && head < (uint32_t)A.heads, vec0 + (int64_t)head * A.block_tokens, lane, sg);
  }
}

template <int H>
void launch_rope(const hq_rope_args& a, hipStream_t st) {
  const dim3 grid((a.tiles + 15) / 16), wg(256);
  if (a.x_bf16)
    hipLaunchKernelGGL((hq_rope_kernel<H, true>), grid, wg, 0, st, a);
  else
    hipLaunchKernelGGL((hq_rope_kernel<H, false>), grid, wg, 0, st, a);
}

template <int FMT>
void launch_append(const hq_cache_append_args& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.sides * a.side_groups + (a.q.tiles + 15) / 16), wg(256);
  if (a.x_bf16 && a.per == 4)
    hipLaunchKernelGGL((hq_cache_append_kernel<FMT, true, 4>), grid, wg, 0, st, a);
  else if (a.x_bf16)
    hipLaunchKernelGGL((hq_cache_append_kernel<FMT, true, 1>), grid, wg, 0, st, a);
  else if (a.per == 4)
    hipLaunchKernelGGL((hq_cache_append_kernel<FMT, false, 4>), grid, wg, 0, st, a);
  else
    hipLaunchKernelGGL((hq_cache_append_kernel<FMT, false, 1>), grid, wg, 0, st, a);
}

}  // namespace

int hq_launch_rope_table(const hq_rope_table_args& a, void* stream) {
  const int64_t n = (a.count * a.pairs + 255) / 256;
  hipLaunchKernelGGL(hq_rope_table_kernel, dim3((uint32_t)(n < 65536 ? n : 65536)), dim3(256), 0, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

int hq_launch_rope(const hq_rope_args& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  switch (a.per) {
    case 4: launch_rope<4>(a, st); break;
    case 2: launch_rope<2>(a, st); break;
    default: launch_rope<1>(a, st);
  }
  return (int)hipGetLastError();
}

int hq_launch_cache_append(const hq_cache_append_args& a, int format, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  switch (format) {
    case HQ_INT8: launch_append<kInt8>(a, st); break;
    case HQ_E4M3: launch_append<kE4M3>(a, st); break;
    default: launch_append<kMx>(a, st);
  }
  return (int)hipGetLastError();
}
