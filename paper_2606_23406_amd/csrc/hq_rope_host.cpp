// Host side of rotary positions and of the cache's append: argument checks and
// launches of the entry points that include/hq.h declares for them.
#include "hq_cache_check.h"

namespace {

hq_status fill_turns(const hq_rotary* r, const int32_t* positions, hq_turns* t) {
  if (!r || r->dims <= 0 || r->dims > HQ_TILE || r->dims % 2 != 0 || r->axes < 1 || r->axes > 4 || r->positions <= 0 ||
      (r->interleaved != 0 && r->interleaved != 1))
    return HQ_ERR_INVALID_ARG;
  if (r->dims % 16 != 0 || r->positions > 0x7FFFFFFF) return HQ_ERR_UNSUPPORTED;  // a lane's 8 values turn or stay
  if (!r->table || !aligned(r->table, 16) || (r->axes > 1 && !r->axis)) return HQ_ERR_INVALID_ARG;
  std::memset(t, 0, sizeof(*t));
  t->table = r->table;
  t->pos = positions;
  t->stats = r->stats;
  t->count = (int32_t)r->positions;
  t->pairs = r->dims / 2;
  t->axes = r->axes;
  t->interleaved = r->interleaved;
  t->runs = 1;
  const int run = r->interleaved ? 4 : 8;
  for (int i = 0; r->axis && i < t->pairs; ++i) {
    if (r->axis[i] >= r->axes) return HQ_ERR_INVALID_ARG;
    t->axis[i >> 4] |= (uint32_t)r->axis[i] << (2 * (i & 15));
    if (r->axis[i] != r->axis[i - i % run]) t->runs = 0;
  }
  return HQ_OK;
}

bool positions_ok(const int32_t* p) { return p && aligned(p, 4); }

// Rows of `heads` head vectors through `t`; rows above 0 and checked.
void fill_rows(const hq_turns& t, const void* x, int32_t xt, int64_t ldx, int64_t rows, int32_t heads, void* y, int32_t yt,
               int64_t ldy, int32_t else_per, hq_rope_args* a) {
  std::memset(a, 0, sizeof(*a));
  a->turn = t;
  a->x = x;
  a->y = y;
  a->ldx = ldx;
  a->ldy = ldy;
  a->heads = heads;
  a->per = hq_rope_per(heads, else_per);
  a->groups = (heads + a->per - 1) / a->per;
  a->tiles = (uint32_t)(rows * a->groups);
  a->by_groups = hq_divide_by((uint32_t)a->groups);
  a->x_bf16 = xt == HQ_BF16;
  a->y_bf16 = yt == HQ_BF16;
  a->past = rows * heads * HQ_TILE * (yt == HQ_BF16 ? 2 : 4) >= HQ_ROPE_PAST;
}

// A row turned in place has to be the same row: each value is read before its own place, and
// no other, is written.
bool in_place_ok(const void* x, int32_t xt, int64_t ldx, const void* y, int32_t yt, int64_t ldy) {
  return x != y || (xt == yt && ldx == ldy);
}

}  // namespace

extern "C" {

hq_status hq_rope_table(const double* freqs, int32_t pairs, int64_t positions, float factor, float* table, void* stream) {
  if (pairs <= 0 || positions < 0 || !std::isfinite(factor)) return HQ_ERR_INVALID_ARG;
  if (pairs > HQ_TILE / 2 || positions > 0x7FFFFFFF) return HQ_ERR_UNSUPPORTED;
  if (positions == 0) return HQ_OK;
  if (!freqs || !aligned(freqs, 8) || !table || !aligned(table, 16)) return HQ_ERR_INVALID_ARG;
  const hq_rope_table_args a = {freqs, table, positions, pairs, factor};
  return hip_status(hq_launch_rope_table(a, stream));
}

hq_status hq_rope(const hq_rotary* r, const void* x, int32_t xt, int64_t ldx, int64_t rows, int32_t heads,
                  const int32_t* positions, int32_t transposed, void* y, int32_t yt, int64_t ldy, void* stream) {
  hq_turns t;
  const hq_status st = fill_turns(r, positions, &t);
  if (st != HQ_OK) return st;
  if (!float_type(xt) || !float_type(yt) || rows < 0 || heads <= 0 || (transposed != 0 && transposed != 1))
    return HQ_ERR_INVALID_ARG;
  if (heads > 1 << 21 || rows > kMaxTiles / heads) return HQ_ERR_UNSUPPORTED;
  if (rows == 0) return HQ_OK;
  const int64_t width = (int64_t)heads * HQ_TILE;
  if (!positions_ok(positions) || !rows_ok(x, xt, ldx, width) || !rows_ok(y, yt, ldy, width) ||
      !in_place_ok(x, xt, ldx, y, yt, ldy))
    return HQ_ERR_INVALID_ARG;
  hq_rope_args a;
  fill_rows(t, x, xt, ldx, rows, heads, y, yt, ldy, 2, &a);
  a.transposed = transposed;
  if ((a.tiles + 15) / 16 > (uint32_t)kMaxGroups) return HQ_ERR_UNSUPPORTED;
  return hip_status(hq_launch_rope(a, stream));
}

hq_status hq_cache_append(hq_plan_t kp, const void* k, int64_t ldk, const hq_cache* kc, hq_plan_t vp, const void* v,
                          int64_t ldv, const hq_cache* vc, int32_t xt, int64_t rows, const int64_t* slots,
                          const hq_rotary* r, const int32_t* positions, const void* q, int64_t ldq, int32_t heads_q,
                          void* q_out, int32_t qot, int64_t ldqo, void* stream) {
  hq_status st = check_sides(kp, kc, vp, v, vc);
  if (st != HQ_OK) return st;
  hq_cache_append_args a;
  std::memset(&a, 0, sizeof(a));
  if ((st = fill_turns(r, positions, &a.turn)) != HQ_OK) return st;
  const bool both = vc != nullptr;
  if (!float_type(xt) || rows < 0 || heads_q < 0 || (heads_q && !float_type(qot))) return HQ_ERR_INVALID_ARG;
  if (heads_q > 1 << 21 || rows > kMaxTiles / kc->heads || (heads_q && rows > kMaxTiles / heads_q))
    return HQ_ERR_UNSUPPORTED;
  if (rows == 0) return HQ_OK;  // no rows need no addresses
  if ((!q != !q_out) || (!q != !heads_q)) return HQ_ERR_INVALID_ARG;
  const int64_t width = (int64_t)kc->heads * HQ_TILE, width_q = (int64_t)heads_q * HQ_TILE;
  if (!slots || !aligned(slots, 8) || !positions_ok(positions) || !rows_ok(k, xt, ldk, width) ||
      (both && !rows_ok(v, xt, ldv, width)))
    return HQ_ERR_INVALID_ARG;
  if (q && (!rows_ok(q, xt, ldq, width_q) || !rows_ok(q_out, qot, ldqo, width_q) || !in_place_ok(q, xt, ldq, q_out, qot, ldqo)))
    return HQ_ERR_INVALID_ARG;
  if ((st = check_device(kp)) != HQ_OK || (both && (st = check_device(vp)) != HQ_OK)) return st;
  fill_side(kp, kc, k, ldk, &a.side[0]);
  if (both) fill_side(vp, vc, v, ldv, &a.side[1]);
  a.sides = both ? 2 : 1;
  a.slots = slots;
  a.heads = kc->heads;
  a.per = hq_rope_per(kc->heads, 1);
  a.groups = (kc->heads + a.per - 1) / a.per;
  a.tiles = (uint32_t)(rows * a.groups);
  a.by_groups = hq_divide_by((uint32_t)a.groups);
  a.block_tokens = kc->block_tokens;
  a.by_block = hq_divide_by((uint32_t)kc->block_tokens);
  a.x_bf16 = xt == HQ_BF16;
  a.side_groups = (a.tiles + 15) / 16;
  if (q) fill_rows(a.turn, q, xt, ldq, rows, heads_q, q_out, qot, ldqo, 1, &a.q);
  if ((int64_t)a.sides * a.side_groups + (a.q.tiles + 15) / 16 > kMaxGroups) return HQ_ERR_UNSUPPORTED;
  return hip_status(hq_launch_cache_append(a, kc->format, stream));
}

}  // extern "C"
