// gfx950 kernel of the RMS norm fused with the 8-bit activation prep
// (hq_rmsnorm_act_prep, hq_rmsnorm_act_prep_fp8).
#include <hip/hip_runtime.h>

#include "hq_device.h"

#pragma clang fp contract(off)

namespace {

// One workgroup per token row, every value in registers from its load to its code.
// 1 / rms(h) is one positive factor of the whole row, so the codes round(y top /
// max|y|) do not depend on it: y is formed from h * w alone, and the factor enters
// s_x = max|y| / (top rms).  So the sum of squares and the maximum meet at one
// barrier, and a row is read once and written once.
// Blocks of 512 columns: up to tile 512 wave w takes the blocks 4 i + w; LONG (tiles of
// 1024 and 2048, two or four blocks) groups of four, 16 (i / 4) + 4 w + i % 4, so that a
// tile lies inside one wave.
template <int NIT, bool FP8, bool LONG>
__global__ __launch_bounds__(256) void hq_norm_prep_kernel(hq_norm_args A) {
  __shared__ float s_max[4], s_sum[4];
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t wave = readfirst((uint32_t)(tid >> 6));
  const int64_t row = blockIdx.x;
  const uint32_t K = (uint32_t)A.K;
  const uint16_t* xrow = (const uint16_t*)A.x + row * A.ldx + 8 * lane;
  const uint16_t* rrow = A.residual ? (const uint16_t*)A.residual + row * A.ldr + 8 * lane : nullptr;
  uint16_t* hrow = A.h ? (uint16_t*)A.h + row * A.ldh + 8 * lane : nullptr;
  auto base_of = [&](int i) -> uint32_t {
    return HQ_SUB * (LONG ? 16u * (i / 4) + 4u * wave + (i & 3) : 4u * i + wave);
  };
  uint4 raw[NIT], res[NIT];
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    const uint32_t base = base_of(i);
    if (base < K) {
      raw[i] = *(const uint4*)(xrow + base);
      if (rrow) res[i] = *(const uint4*)(rrow + base);
    }
  }
  const XSigns sg(lane);
  float v[NIT][8], amax = 0.0f, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    const uint32_t base = base_of(i);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
    if (base >= K) continue;
    uint32_t w4[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    if (rrow) {
      const uint32_t r4[4] = {res[i].x, res[i].y, res[i].z, res[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)  // h is the bf16 that is stored, and what the norm is of
        w4[e] = cvt_pk_bf16(__uint_as_float(w4[e] << 16) + __uint_as_float(r4[e] << 16),
                            __uint_as_float(w4[e] & 0xFFFF0000u) + __uint_as_float(r4[e] & 0xFFFF0000u));
    }
    if (hrow) *(uint4*)(hrow + base) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
    float wt[8];
    const uint32_t col = base + 8 * lane;
    if (A.w_bf16) {
      const uint4 x = *(const uint4*)((const uint16_t*)A.weight + col);
      const uint32_t x4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        wt[2 * e] = __uint_as_float(x4[e] << 16);
        wt[2 * e + 1] = __uint_as_float(x4[e] & 0xFFFF0000u);
      }
    } else {
      const float4 a = *(const float4*)((const float*)A.weight + col);
      const float4 b = *(const float4*)((const float*)A.weight + col + 4);
      wt[0] = a.x; wt[1] = a.y; wt[2] = a.z; wt[3] = a.w;
      wt[4] = b.x; wt[5] = b.y; wt[6] = b.z; wt[7] = b.w;
    }
    const uint32_t dbits = sign_bits8(A.dmask, col);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = __uint_as_float(w4[e] << 16), b = __uint_as_float(w4[e] & 0xFFFF0000u);
      sum = __builtin_fmaf(a, a, sum);
      sum = __builtin_fmaf(b, b, sum);
      v[i][2 * e] = flip(a * wt[2 * e], dbits, 2 * e);
      v[i][2 * e + 1] = flip(b * wt[2 * e + 1], dbits, 2 * e + 1);
    }
    fwht128(v[i], sg);
    if (LONG || A.tile >= 256) {
      const float s = (lane & 16) ? -1.0f : 1.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf(v[i][e], s, swz_xor16(v[i][e]));
    }
    if (LONG || A.tile >= 512) {
      const float s = (lane & 32) ? -1.0f : 1.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf(v[i][e], s, lane_xor32(v[i][e]));
    }
  }
  if constexpr (LONG) {
#pragma unroll
    for (int h = 1; h <= 2; h <<= 1) {
      if (h == 2 && A.tile < 2048) break;
#pragma unroll
      for (int i = 0; i < NIT; ++i)
        if ((i & h) == 0)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float a = v[i][e], b = v[i + h][e];
            v[i][e] = a + b;
            v[i + h][e] = a - b;
          }
    }
  }
#pragma unroll
  for (int i = 0; i < NIT; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = __builtin_fmaxf(amax, __builtin_fabsf(v[i][e]));
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    amax = __builtin_fmaxf(amax, __shfl_xor(amax, m, 64));
    sum += __shfl_xor(sum, m, 64);
  }
  if (lane == 0) {
    s_max[wave] = amax;
    s_sum[wave] = sum;
  }
  __syncthreads();
  amax = __builtin_fmaxf(__builtin_fmaxf(s_max[0], s_max[1]), __builtin_fmaxf(s_max[2], s_max[3]));
  const float top = FP8 ? 448.0f : 127.0f;  // E4M3's largest magnitude, or int8's
  // below 2^-100 the reciprocal could overflow: such a row counts as zeros
  const float inv = amax < 0x1p-100f ? 0.0f : top / amax;
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    const uint32_t base = base_of(i);
    if (base >= K) continue;
    uint32_t packed[2] = {0u, 0u};
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[e] = v[i][e] * inv;
      if (!FP8) q[e] = __builtin_rintf(q[e]);
      q[e] = __builtin_fminf(__builtin_fmaxf(q[e], -top), top);
    }
    if constexpr (FP8) {
      packed[0] = e4m3x4(q[0], q[1], q[2], q[3]);
      packed[1] = e4m3x4(q[4], q[5], q[6], q[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) packed[e >> 2] |= ((uint32_t)(int32_t)q[e] & 0xFFu) << (8 * (e & 3));
    }
    *(uint2*)(A.xq + row * A.K + base + 8 * lane) = make_uint2(packed[0], packed[1]);
  }
  if (tid == 0) {
    const float mean = ((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) / (float)A.K;
    const float rms = __builtin_sqrtf(mean + A.eps);
    // a NaN or an infinity anywhere in the row makes its scale NaN
    A.sx[row] = rms <= 3.4028234663852886e38f ? amax < 0x1p-100f ? 0.0f : amax / top / rms : __builtin_nanf("");
  }
}

}  // namespace

template <bool FP8>
static void launch(const hq_norm_args& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.M), wg(256);
  if (a.tile > HQ_SUB) {
    if (a.K <= 8192)
      hipLaunchKernelGGL((hq_norm_prep_kernel<4, FP8, true>), grid, wg, 0, st, a);
    else
      hipLaunchKernelGGL((hq_norm_prep_kernel<8, FP8, true>), grid, wg, 0, st, a);
  } else if (a.K <= 2048) {
    hipLaunchKernelGGL((hq_norm_prep_kernel<1, FP8, false>), grid, wg, 0, st, a);
  } else if (a.K <= 4096) {
    hipLaunchKernelGGL((hq_norm_prep_kernel<2, FP8, false>), grid, wg, 0, st, a);
  } else if (a.K <= 8192) {
    hipLaunchKernelGGL((hq_norm_prep_kernel<4, FP8, false>), grid, wg, 0, st, a);
  } else {
    hipLaunchKernelGGL((hq_norm_prep_kernel<8, FP8, false>), grid, wg, 0, st, a);
  }
}

int hq_launch_norm_prep(const hq_norm_args& a, void* stream) {
  if (a.fp8)
    launch<true>(a, (hipStream_t)stream);
  else
    launch<false>(a, (hipStream_t)stream);
  return (int)hipGetLastError();
}
