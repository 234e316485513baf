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
// barrier, and a row is read once and written once: memory bounds it.  8192 x 4096 with a
// residual takes 46.7 us (5.0 TB/s), 4000 x 14336 76.6 (5.25), as a large copy; 1000 rows, two
// rounds of workgroups, 60 % of that.
// Blocks of 512 columns: up to tile 512 wave w of W takes the blocks W i + w; LONG (tiles
// of 1024 and 2048, two or four blocks) groups of four, 4 W (i / 4) + 4 w + i % 4, so that
// a tile lies inside one wave.
template <int W, int NIT, bool FP8, bool LONG>
__global__ __launch_bounds__(64 * W) void hq_norm_prep_kernel(hq_norm_args A) {
  __shared__ float s_max[W], s_sum[W];
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t wave = readfirst((uint32_t)(tid >> 6));
  const int64_t row = blockIdx.x;
  const uint32_t K = (uint32_t)A.K;
  const uint16_t* xrow = (const uint16_t*)A.x + row * A.ldx + 8 * lane;
  const uint16_t* rrow = A.residual ? (const uint16_t*)A.residual + row * A.ldr + 8 * lane : nullptr;
  uint16_t* hrow = A.h ? (uint16_t*)A.h + row * A.ldh + 8 * lane : nullptr;
  auto base_of = [&](int i) -> uint32_t {
    return HQ_SUB * (LONG ? 4u * W * (i / 4) + 4u * wave + (i & 3) : (uint32_t)W * i + wave);
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
  const TwSigns sg(lane);  // the transform leaves sigma times the values
  const float s16 = (lane & 16) ? -1.0f : 1.0f, s32 = (lane & 32) ? -1.0f : 1.0f;
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
    const uint4 dw = *(const uint4*)(A.dsign16 + (col >> 1));
    const uint32_t d4[4] = {dw.x, dw.y, dw.z, dw.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = w4[e] ^ d4[e];
      const float a = __uint_as_float(x << 16), b = __uint_as_float(x & 0xFFFF0000u);
      sum = __builtin_fmaf(a, a, sum);
      sum = __builtin_fmaf(b, b, sum);
      v[i][2 * e] = a * wt[2 * e];
      v[i][2 * e + 1] = b * wt[2 * e + 1];
    }
    fwht128_tw(v[i], sg);
    if (LONG || A.tile >= 256) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf(v[i][e], s16, swz_xor16(v[i][e]));
    }
    if (LONG || A.tile >= 512) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf(v[i][e], s32, lane_xor32(v[i][e]));
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
    for (int e = 0; e < 8; ++e) amax = __builtin_elementwise_maximum(amax, __builtin_fabsf(v[i][e]));
  amax = __builtin_elementwise_maximum(amax, dpp_xor<1>(amax));
  sum += dpp_xor<1>(sum);
  amax = __builtin_elementwise_maximum(amax, dpp_xor<2>(amax));
  sum += dpp_xor<2>(sum);
  amax = __builtin_elementwise_maximum(amax, swz_xor4(amax));
  sum += swz_xor4(sum);
  amax = __builtin_elementwise_maximum(amax, dpp_xor<8>(amax));
  sum += dpp_xor<8>(sum);
  amax = __builtin_elementwise_maximum(amax, swz_xor16(amax));
  sum += swz_xor16(sum);
  amax = __builtin_elementwise_maximum(amax, lane_xor32(amax));
  sum += lane_xor32(sum);
  if (lane == 0) {
    s_max[wave] = amax;
    s_sum[wave] = sum;
  }
  __syncthreads();
  amax = s_max[0];
  sum = s_sum[0];
#pragma unroll
  for (int x = 1; x < W; ++x) {
    amax = __builtin_elementwise_maximum(amax, s_max[x]);
    sum += s_sum[x];
  }
  const float top = FP8 ? 448.0f : 127.0f;  // E4M3's largest magnitude, or int8's
  // below 2^-100 the reciprocal could overflow: such a row counts as zeros
  const float inv = amax < 0x1p-100f ? 0.0f : xor_sign(top / amax, sg.sigma);
  // |v inv| is top (1 + 2^-23) at most, which rounds to top in both formats: no clamp.
  // (A row with a NaN has the scale NaN, whatever its codes.)
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    const uint32_t base = base_of(i);
    if (base >= K) continue;
    uint2 packed;
    if constexpr (FP8) {
      packed.x = e4m3x4(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
      packed.y = e4m3x4(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
    } else {
      packed = int8x8(v[i], inv);
    }
    *(uint2*)(A.xq + row * A.K + base + 8 * lane) = packed;
  }
  if (tid == 0) {
    const float rms = __builtin_sqrtf(sum / (float)A.K + A.eps);
    // a NaN or an infinity anywhere in h, h * weight or the transform makes the row's scale
    // NaN (the maximum keeps a NaN)
    constexpr float most = 3.4028234663852886e38f;
    A.sx[row] = !(rms <= most && amax <= most) ? __builtin_nanf("") : amax < 0x1p-100f ? 0.0f : amax / top / rms;
  }
}

}  // namespace

template <int W, int NIT, bool FP8, bool LONG>
static void launch(const hq_norm_args& a, hipStream_t st) {
  hipLaunchKernelGGL((hq_norm_prep_kernel<W, NIT, FP8, LONG>), dim3((uint32_t)a.M), dim3(64 * W), 0, st, a);
}

// Two blocks a wave, as many waves as that takes.  More blocks a wave leave less
// in flight (1000 x 14336 at tile 512 without a residual: 16.4 us with 8 blocks on
// four waves, 14.7 with 4 on eight, 14.2 with 2 on sixteen; 4000 x 8192 with one
// 49.4, 46.7 and -), fewer make the barrier's share larger (8192 x 4096: 46.8 us with
// 2 on four, 48.2 with 1 on eight).
template <bool FP8>
static void launch(const hq_norm_args& a, hipStream_t st) {
  if (a.tile > HQ_SUB) {
    if (a.K <= 8192)
      launch<4, 4, FP8, true>(a, st);
    else
      launch<8, 4, FP8, true>(a, st);
  } else if (a.K <= 2048) {
    launch<4, 1, FP8, false>(a, st);
  } else if (a.K <= 4096) {
    launch<4, 2, FP8, false>(a, st);
  } else if (a.K <= 8192) {
    launch<8, 2, FP8, false>(a, st);
  } else {
    launch<16, 2, FP8, false>(a, st);
  }
}

int hq_launch_norm_prep(const hq_norm_args& args, void* stream) {
  // a grid holds less than 2^32 threads: at most 2^21 rows of 1024 a launch
  constexpr int64_t kRows = (int64_t)1 << 21;
  hq_norm_args a = args;
  for (int64_t left = args.M; left > 0; left -= kRows) {
    a.M = left < kRows ? left : kRows;
    if (a.fp8)
      launch<true>(a, (hipStream_t)stream);
    else
      launch<false>(a, (hipStream_t)stream);
    if (const hipError_t e = hipGetLastError()) return (int)e;
    a.x = (const uint16_t*)a.x + kRows * a.ldx;
    if (a.residual) a.residual = (const uint16_t*)a.residual + kRows * a.ldr;
    if (a.h) a.h = (uint16_t*)a.h + kRows * a.ldh;
    a.xq += kRows * a.K;
    a.sx += kRows;
  }
  return 0;
}
