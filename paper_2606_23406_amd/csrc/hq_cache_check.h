// Argument checks that the host sides of the cache's entry points share, and what its
// one-token attentions hand to their launch.
#ifndef HQ_CACHE_CHECK_H
#define HQ_CACHE_CHECK_H
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

// The caches of a write: of keys alone, or of keys and values that are written together.
hq_status check_sides(const hq_plan_s* kp, const hq_cache* kc, const hq_plan_s* vp, const void* v, const hq_cache* vc) {
  hq_status st = check_cache(kp, kc);
  if (st != HQ_OK) return st;
  if (!vc) return v ? HQ_ERR_INVALID_ARG : HQ_OK;
  if ((st = check_cache(vp, vc)) != HQ_OK) return st;
  if (vc->format != kc->format || vc->heads != kc->heads || vc->block_tokens != kc->block_tokens)
    return HQ_ERR_INVALID_ARG;
  if (vc->codes == kc->codes || vc->scales == kc->scales) return HQ_ERR_INVALID_ARG;
  return HQ_OK;
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

// What every attention over a cache checks and hands on: `rows` queries of `batch` sequences.
// *run: there is anything to do.
hq_status attention_args(const hq_plan_s* kp, const hq_cache* k, const hq_plan_s* vp, const hq_cache* v, const void* q,
                         int32_t qt, int64_t batch, int64_t rows, int32_t heads_q, float scale,
                         const int32_t* block_table, int32_t max_blocks, const int32_t* seq_lens, int32_t window,
                         int32_t sinks, void* out, int32_t ot, hq_cache_attn_args* a, bool* run) {
  *run = false;
  hq_status st = check_cache(kp, k);
  if (st != HQ_OK || (st = check_cache(vp, v)) != HQ_OK) return st;
  if (v->format != k->format || v->heads != k->heads || v->block_tokens != k->block_tokens || v->blocks != k->blocks)
    return HQ_ERR_INVALID_ARG;
  if (!float_type(qt) || !float_type(ot) || batch < 0 || rows < 0 || heads_q <= 0 || heads_q % k->heads != 0 ||
      max_blocks <= 0 || !std::isfinite(scale))
    return HQ_ERR_INVALID_ARG;
  const int64_t group = heads_q / k->heads;
  if (group > 16) return HQ_ERR_UNSUPPORTED;
  const int64_t max_tokens = (int64_t)max_blocks * k->block_tokens;
  if (max_tokens > (int64_t)1 << 30 || batch > 0x7FFFFFFF / heads_q || rows > 0x7FFFFFFF / heads_q)
    return HQ_ERR_UNSUPPORTED;
  if (batch == 0 || rows == 0) return HQ_OK;
  if (!q || !out || !block_table || !seq_lens || !aligned(q, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4))
    return HQ_ERR_INVALID_ARG;
  std::memset(a, 0, sizeof(*a));
  a->k_codes = (const uint8_t*)k->codes;
  a->k_scales = k->scales;
  a->v_codes = (const uint8_t*)v->codes;
  a->v_scales = v->scales;
  a->k_dsign16 = kp->d_dsign16;
  a->v_dsign16 = vp->d_dsign16;
  a->q = q;
  a->out = out;
  a->table = block_table;
  a->seq_lens = seq_lens;
  a->stats = k->stats;
  a->batch = batch;
  a->blocks = (int32_t)k->blocks;
  a->heads_q = heads_q;
  a->heads_kv = k->heads;
  a->group = (int32_t)group;
  a->max_blocks = max_blocks;
  a->block_tokens = k->block_tokens;
  a->by_block = hq_divide_by((uint32_t)k->block_tokens);
  // no sequence is longer than 2^30 tokens, so no larger window or number of sinks differs
  a->window = window < 1 << 30 ? window : 1 << 30;
  a->sinks = sinks < 1 << 30 ? sinks : 1 << 30;
  a->q_bf16 = qt == HQ_BF16;
  a->out_bf16 = ot == HQ_BF16;
  a->qscale = scale * (1.4426950408889634f / 128.0f);  // log2(e): the softmax runs in base 2
  *run = true;
  return HQ_OK;
}

// Workspace of a one-token attention whose sequences have `seen` tokens at most to look at.
size_t one_token_bytes(const hq_cache* k, int64_t batch, int32_t heads_q, int64_t seen) {
  if (seen <= HQ_CACHE_WHOLE) return 0;
  const int64_t n = hq_cache_items(batch, k->heads, seen) * heads_q;
  return (size_t)n * (HQ_TILE + 2) * sizeof(float) + (size_t)batch * sizeof(hq_cache_of) +
         (size_t)(hq_cache_joins(batch, k->heads) + 1) * sizeof(int32_t);
}

hq_status one_token(const hq_plan_s* kp, const hq_cache* k, const hq_plan_s* vp, hq_cache_attn_args& a, void* workspace,
                    size_t ws_bytes, void* stream) {
  const int64_t seen = hq_cache_seen((int64_t)a.max_blocks * a.block_tokens, a.window, a.sinks, 0);
  a.items = hq_cache_items(a.batch, a.heads_kv, seen);
  a.joins = hq_cache_joins(a.batch, a.heads_kv);
  a.join = seen > HQ_CACHE_WHOLE;
  if (a.items * a.heads_q > 0x7FFFFFFF || a.items * a.heads_kv > kMaxGroups) return HQ_ERR_UNSUPPORTED;
  if (a.join && (!workspace || !aligned(workspace, 16) || ws_bytes < one_token_bytes(k, a.batch, a.heads_q, seen)))
    return HQ_ERR_INVALID_ARG;
  hq_status st = check_device(kp);
  if (st != HQ_OK || (st = check_device(vp)) != HQ_OK) return st;
  if (a.join) {
    const int64_t n = a.items * a.heads_q;
    a.part_acc = (float*)workspace;
    a.part_m = a.part_acc + n * HQ_TILE;
    a.part_l = a.part_m + n;
    a.parts = (hq_cache_of*)(a.part_l + n);
    a.split = (int32_t*)(a.parts + a.batch);
  }
  return hip_status(hq_launch_cache_attention(a, k->format, stream));
}

}  // namespace

#endif
