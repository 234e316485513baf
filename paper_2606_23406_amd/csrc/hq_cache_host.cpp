// Host side of the fixed-rate key-value cache and of the fused norm: argument
// checks and launches of the entry points that include/hq.h declares for them.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "hq_cache_check.h"

namespace {

hq_status norm_prep(hq_plan_t p, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                    int32_t wt, float eps, int64_t M, void* h, int64_t ldh, int8_t* xq, float* sx, int fp8,
                    void* stream) {
  if (!p || M < 0 || !float_type(wt) || !(eps > 0.0f) || !std::isfinite(eps)) return HQ_ERR_INVALID_ARG;
  if (p->cols > 16384 || M > 0x7FFFFFFF) return HQ_ERR_UNSUPPORTED;
  if (M == 0) return HQ_OK;
  if (!rows_ok(x, HQ_BF16, ldx, p->cols) || !weight || !aligned(weight, 16) || !xq || !aligned(xq, 8) || !sx)
    return HQ_ERR_INVALID_ARG;
  if (residual && !rows_ok(residual, HQ_BF16, ldr, p->cols)) return HQ_ERR_INVALID_ARG;
  if (h && !rows_ok(h, HQ_BF16, ldh, p->cols)) return HQ_ERR_INVALID_ARG;
  const hq_status st = check_device(p);
  if (st != HQ_OK) return st;
  hq_norm_args a;
  std::memset(&a, 0, sizeof(a));
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.h = h;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldh = ldh;
  a.M = M;
  a.K = p->cols;
  a.xq = xq;
  a.sx = sx;
  a.dsign16 = p->d_dsign16;
  a.eps = eps;
  a.w_bf16 = wt == HQ_BF16;
  a.fp8 = fp8;
  a.tile = p->tile;
  return hip_status(hq_launch_norm_prep(a, stream));
}

}  // namespace

extern "C" {

hq_status hq_cache_write(hq_plan_t kp, const void* k, int64_t ldk, const hq_cache* kc, hq_plan_t vp, const void* v,
                         int64_t ldv, const hq_cache* vc, int32_t xt, int64_t rows, const int64_t* slots,
                         void* stream) {
  hq_status st = check_sides(kp, kc, vp, v, vc);
  if (st != HQ_OK) return st;
  const bool both = vc != nullptr;
  if (!float_type(xt) || rows < 0) return HQ_ERR_INVALID_ARG;
  if (rows > kMaxTiles / kc->heads) return HQ_ERR_UNSUPPORTED;
  if (rows == 0) return HQ_OK;
  const int64_t width = (int64_t)kc->heads * HQ_TILE;
  if (!slots || !aligned(slots, 8) || !rows_ok(k, xt, ldk, width) || (both && !rows_ok(v, xt, ldv, width)))
    return HQ_ERR_INVALID_ARG;
  if ((st = check_device(kp)) != HQ_OK || (both && (st = check_device(vp)) != HQ_OK)) return st;
  hq_cache_io_args a;
  std::memset(&a, 0, sizeof(a));
  fill_side(kp, kc, k, ldk, &a.side[0]);
  if (both) fill_side(vp, vc, v, ldv, &a.side[1]);
  a.slots = slots;
  a.tiles = (uint32_t)(rows * kc->heads);
  a.heads = kc->heads;
  a.block_tokens = kc->block_tokens;
  a.by_heads = hq_divide_by((uint32_t)kc->heads);
  a.by_block = hq_divide_by((uint32_t)kc->block_tokens);
  a.x_bf16 = xt == HQ_BF16;
  return hip_status(hq_launch_cache_write(a, kc->format, both ? 2 : 1, stream));
}

hq_status hq_cache_read(hq_plan_t p, const hq_cache* c, const int64_t* slots, int64_t rows, void* y, int32_t yt,
                        int64_t ld, void* stream) {
  hq_status st = check_cache(p, c);
  if (st != HQ_OK) return st;
  if (!float_type(yt) || rows < 0) return HQ_ERR_INVALID_ARG;
  if (rows > kMaxTiles / c->heads) return HQ_ERR_UNSUPPORTED;
  if (rows == 0) return HQ_OK;
  if (!slots || !aligned(slots, 8) || !rows_ok(y, yt, ld, (int64_t)c->heads * HQ_TILE)) return HQ_ERR_INVALID_ARG;
  if ((st = check_device(p)) != HQ_OK) return st;
  hq_cache_io_args a;
  std::memset(&a, 0, sizeof(a));
  fill_side(p, c, nullptr, 0, &a.side[0]);
  a.slots = slots;
  a.tiles = (uint32_t)(rows * c->heads);
  a.heads = c->heads;
  a.block_tokens = c->block_tokens;
  a.by_heads = hq_divide_by((uint32_t)c->heads);
  a.by_block = hq_divide_by((uint32_t)c->block_tokens);
  a.y = y;
  a.ldy = ld;
  a.y_bf16 = yt == HQ_BF16;
  return hip_status(hq_launch_cache_read(a, c->format, stream));
}

size_t hq_cache_attention_workspace_bytes(const hq_cache* k, int64_t batch, int32_t heads_q, int32_t max_blocks) {
  if (!k || batch <= 0 || heads_q <= 0 || max_blocks <= 0 || k->heads <= 0 || k->block_tokens <= 0 ||
      heads_q % k->heads != 0)
    return 0;
  return one_token_bytes(k, batch, heads_q, (int64_t)max_blocks * k->block_tokens);
}

hq_status hq_cache_attention(hq_plan_t kp, const hq_cache* k, hq_plan_t vp, const hq_cache* v, const void* q,
                             int32_t qt, int64_t batch, int32_t heads_q, float scale, const int32_t* block_table,
                             int32_t max_blocks, const int32_t* seq_lens, void* out, int32_t ot, void* workspace,
                             size_t ws_bytes, void* stream) {
  hq_cache_attn_args a;
  bool run;
  const hq_status st = attention_args(kp, k, vp, v, q, qt, batch, batch, heads_q, scale, block_table, max_blocks, seq_lens,
                                      0, 0, out, ot, &a, &run);
  if (st != HQ_OK || !run) return st;
  return one_token(kp, k, vp, a, workspace, ws_bytes, stream);
}

hq_status hq_rmsnorm_act_prep(hq_plan_t p, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                              const void* weight, int32_t wt, float eps, int64_t M, void* h, int64_t ldh, int8_t* xq,
                              float* sx, void* stream) {
  return norm_prep(p, x, ldx, residual, ldr, weight, wt, eps, M, h, ldh, xq, sx, 0, stream);
}

hq_status hq_rmsnorm_act_prep_fp8(hq_plan_t p, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                  const void* weight, int32_t wt, float eps, int64_t M, void* h, int64_t ldh,
                                  uint8_t* xq, float* sx, void* stream) {
  return norm_prep(p, x, ldx, residual, ldr, weight, wt, eps, M, h, ldh, (int8_t*)xq, sx, 1, stream);
}

}  // extern "C"
