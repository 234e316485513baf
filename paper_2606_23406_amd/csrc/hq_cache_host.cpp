// Host side of the fixed-rate key-value cache and of the fused norm: argument
// checks and launches of the entry points that include/hq.h declares for them.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "hq_internal.h"

namespace {

hq_status hip_status(int e) { return e == 0 ? HQ_OK : HQ_ERR_HIP; }

// A grid holds less than 2^32 threads: 2^24 workgroups of 256 less one, and of a cache's
// vectors, 32 a workgroup, 2^28 with room to spare.
constexpr int64_t kMaxGroups = (1 << 24) - 1, kMaxTiles = 1 << 28;

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The plan gives the cache its signs only: tile 128, no KV option (a stored
// vector is the cast of H D x alone), enough columns for the cache's heads, and
// its constants on the current device.
hq_status check_cache(const hq_plan_s* p, const hq_cache* c) {
  if (!p || !c) return HQ_ERR_INVALID_ARG;
  if (p->tile != HQ_TILE || p->rotation != HQ_ROT_NONE || p->dither || p->norm_fp16) return HQ_ERR_UNSUPPORTED;
  if (c->format != HQ_INT8 && c->format != HQ_E4M3 && c->format != HQ_MXFP4) return HQ_ERR_INVALID_ARG;
  if (c->heads <= 0 || (int64_t)c->heads * HQ_TILE > p->cols || c->blocks <= 0 || c->block_tokens <= 0)
    return HQ_ERR_INVALID_ARG;
  if (c->block_tokens % 16 != 0 || c->block_tokens > 1 << 24) return HQ_ERR_UNSUPPORTED;  // 32-bit bytes of a block
  if (c->blocks > 0x7FFFFFFF / c->block_tokens) return HQ_ERR_UNSUPPORTED;  // slots are 31-bit
  if (!c->codes || !c->scales || !aligned(c->codes, 16) || !aligned(c->scales, 16)) return HQ_ERR_INVALID_ARG;
  return HQ_OK;
}

hq_status check_device(const hq_plan_s* p) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return HQ_ERR_HIP;
  return dev == p->device ? HQ_OK : HQ_ERR_INVALID_ARG;
}

bool float_type(int32_t t) { return t == HQ_BF16 || t == HQ_FP32; }

// Rows of heads * 128 values in 16-byte pieces.
bool rows_ok(const void* p, int32_t type, int64_t ld, int64_t width) {
  return p && aligned(p, 16) && ld >= width && ld % (type == HQ_BF16 ? 8 : 4) == 0;
}

void fill_side(const hq_plan_s* p, const hq_cache* c, const void* x, int64_t ld, hq_cache_side* s) {
  s->x = x;
  s->ld = ld;
  s->codes = (uint8_t*)c->codes;
  s->scales = c->scales;
  s->slots = c->blocks * c->block_tokens;
  s->dsign16 = p->d_dsign16;
  s->stats = c->stats;
}

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
  hq_status st = check_cache(kp, kc);
  if (st != HQ_OK) return st;
  const bool both = vc != nullptr;
  if (both) {
    if ((st = check_cache(vp, vc)) != HQ_OK) return st;
    if (vc->format != kc->format || vc->heads != kc->heads || vc->block_tokens != kc->block_tokens)
      return HQ_ERR_INVALID_ARG;
    if (vc->codes == kc->codes || vc->scales == kc->scales) return HQ_ERR_INVALID_ARG;
  } else if (v) {
    return HQ_ERR_INVALID_ARG;
  }
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
  const int64_t max_tokens = (int64_t)max_blocks * k->block_tokens;
  if (max_tokens <= HQ_CACHE_WHOLE) return 0;
  const int64_t n = hq_cache_items(batch, k->heads, max_tokens) * heads_q;
  return (size_t)n * (HQ_TILE + 2) * sizeof(float) + (size_t)batch * sizeof(hq_cache_of) +
         (size_t)(hq_cache_joins(batch, k->heads) + 1) * sizeof(int32_t);
}

hq_status hq_cache_attention(hq_plan_t kp, const hq_cache* k, hq_plan_t vp, const hq_cache* v, const void* q,
                             int32_t qt, int64_t batch, int32_t heads_q, float scale, const int32_t* block_table,
                             int32_t max_blocks, const int32_t* seq_lens, void* out, int32_t ot, void* workspace,
                             size_t ws_bytes, void* stream) {
  hq_status st = check_cache(kp, k);
  if (st != HQ_OK || (st = check_cache(vp, v)) != HQ_OK) return st;
  if (v->format != k->format || v->heads != k->heads || v->block_tokens != k->block_tokens || v->blocks != k->blocks)
    return HQ_ERR_INVALID_ARG;
  if (!float_type(qt) || !float_type(ot) || batch < 0 || heads_q <= 0 || heads_q % k->heads != 0 ||
      max_blocks <= 0 || !std::isfinite(scale))
    return HQ_ERR_INVALID_ARG;
  const int64_t group = heads_q / k->heads;
  if (group > 16) return HQ_ERR_UNSUPPORTED;
  const int64_t max_tokens = (int64_t)max_blocks * k->block_tokens;
  if (max_tokens > (int64_t)1 << 30 || batch > 0x7FFFFFFF / heads_q) return HQ_ERR_UNSUPPORTED;
  if (batch == 0) return HQ_OK;
  if (!q || !out || !block_table || !seq_lens || !aligned(q, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4))
    return HQ_ERR_INVALID_ARG;
  const int64_t items = hq_cache_items(batch, k->heads, max_tokens);
  const bool join = max_tokens > HQ_CACHE_WHOLE;
  if (items * heads_q > 0x7FFFFFFF || items * k->heads > kMaxGroups) return HQ_ERR_UNSUPPORTED;
  if (join && (!workspace || !aligned(workspace, 16) ||
               ws_bytes < hq_cache_attention_workspace_bytes(k, batch, heads_q, max_blocks)))
    return HQ_ERR_INVALID_ARG;
  if ((st = check_device(kp)) != HQ_OK || (st = check_device(vp)) != HQ_OK) return st;
  hq_cache_attn_args a;
  std::memset(&a, 0, sizeof(a));
  a.k_codes = (const uint8_t*)k->codes;
  a.k_scales = k->scales;
  a.v_codes = (const uint8_t*)v->codes;
  a.v_scales = v->scales;
  a.k_dsign16 = kp->d_dsign16;
  a.v_dsign16 = vp->d_dsign16;
  a.q = q;
  a.out = out;
  a.table = block_table;
  a.seq_lens = seq_lens;
  if (join) {
    const int64_t n = items * heads_q;
    a.part_acc = (float*)workspace;
    a.part_m = a.part_acc + n * HQ_TILE;
    a.part_l = a.part_m + n;
    a.parts = (hq_cache_of*)(a.part_l + n);
    a.split = (int32_t*)(a.parts + batch);
  }
  a.stats = k->stats;
  a.batch = batch;
  a.blocks = (int32_t)k->blocks;
  a.heads_q = heads_q;
  a.heads_kv = k->heads;
  a.group = (int32_t)group;
  a.max_blocks = max_blocks;
  a.block_tokens = k->block_tokens;
  a.items = items;
  a.joins = hq_cache_joins(batch, k->heads);
  a.join = join;
  a.q_bf16 = qt == HQ_BF16;
  a.out_bf16 = ot == HQ_BF16;
  a.qscale = scale * (1.4426950408889634f / 128.0f);  // log2(e): the softmax runs in base 2
  return hip_status(hq_launch_cache_attention(a, k->format, stream));
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
