// Host side of the cache's windowed one-token attention and of the attention of
// drafted tokens: argument checks and launches of the entry points that
// include/hq.h declares for them.
#include "hq_cache_check.h"

namespace {

// What a workspace size goes by.
bool sizes_ok(const hq_cache* k, int64_t batch, int32_t heads_q, int32_t max_blocks, int32_t window, int32_t sinks) {
  return k && batch > 0 && heads_q > 0 && max_blocks > 0 && k->heads > 0 && k->block_tokens > 0 &&
         heads_q % k->heads == 0 && window >= 0 && sinks >= 0;
}

struct TreeSize {
  int64_t seen, tile, tiles, items, joins, parts;
  size_t bytes;  // enough for the call, and never less for a larger one
};

// `all`: drafted tokens of all sequences.
TreeSize tree_size(int64_t batch, int64_t all, int32_t heads, int32_t group, int64_t max_tokens, int32_t max_tree,
                   int32_t window, int32_t sinks) {
  TreeSize s;
  const int64_t rows = (int64_t)max_tree * group;
  s.seen = hq_cache_seen(max_tokens, window, sinks, max_tree);
  if (all > batch * max_tree) all = batch * max_tree;  // some are of no sequence
  s.tile = hq_tree_tile(rows, all * group, batch, heads, s.seen);
  s.tiles = (rows + s.tile - 1) / s.tile;
  s.items = hq_tree_items(batch, heads, s.seen, s.tiles);
  s.joins = hq_cache_joins(batch, heads);
  s.parts = s.items * heads * s.tile;
  // a bound on the parts that does not fall from one rule's tiles to another's, nor go by `all`
  const int64_t least = rows <= 16 ? 16 : 4 * rows < 3 * 128 ? 32 : 128, padded = (rows + least - 1) / least * least;
  const int64_t most = (s.seen + HQ_CACHE_LEAST - 1) / HQ_CACHE_LEAST * batch * heads * padded;
  const int64_t even = batch * heads * padded + (HQ_CACHE_WG_TARGET + heads) * least, parts = most < even ? most : even;
  s.bytes = s.seen <= HQ_CACHE_WHOLE ? 0
                                     : (size_t)parts * (HQ_TILE + 2) * sizeof(float) + (size_t)batch * sizeof(hq_cache_of) +
                                           (size_t)(s.joins + 1) * sizeof(int32_t);
  return s;
}

}  // namespace

extern "C" {

size_t hq_cache_window_workspace_bytes(const hq_cache* k, int64_t batch, int32_t heads_q, int32_t max_blocks,
                                       int32_t window, int32_t sinks) {
  if (!sizes_ok(k, batch, heads_q, max_blocks, window, sinks) || window == 0) return 0;
  return one_token_bytes(k, batch, heads_q, hq_cache_seen((int64_t)max_blocks * k->block_tokens, window, sinks, 0));
}

hq_status hq_cache_window_attention(hq_plan_t kp, const hq_cache* k, hq_plan_t vp, const hq_cache* v, const void* q,
                                    int32_t qt, int64_t batch, int32_t heads_q, float scale, const int32_t* block_table,
                                    int32_t max_blocks, const int32_t* seq_lens, int32_t window, int32_t sinks, void* out,
                                    int32_t ot, void* workspace, size_t ws_bytes, void* stream) {
  if (window <= 0 || sinks < 0) return HQ_ERR_INVALID_ARG;
  hq_cache_attn_args a;
  bool run;
  const hq_status st = attention_args(kp, k, vp, v, q, qt, batch, batch, heads_q, scale, block_table, max_blocks, seq_lens,
                                      window, sinks, out, ot, &a, &run);
  if (st != HQ_OK || !run) return st;
  return one_token(kp, k, vp, a, workspace, ws_bytes, stream);
}

size_t hq_cache_tree_workspace_bytes(const hq_cache* k, int64_t batch, int32_t heads_q, int32_t max_blocks,
                                     int32_t max_tree, int32_t window, int32_t sinks) {
  if (!sizes_ok(k, batch, heads_q, max_blocks, window, sinks) || max_tree <= 0 || max_tree > 64) return 0;
  return tree_size(batch, batch * max_tree, k->heads, heads_q / k->heads, (int64_t)max_blocks * k->block_tokens, max_tree,
                   window, sinks)
      .bytes;
}

hq_status hq_cache_tree_attention(hq_plan_t kp, const hq_cache* k, hq_plan_t vp, const hq_cache* v, const void* q,
                                  int32_t qt, int64_t rows, int32_t heads_q, float scale, const uint64_t* masks,
                                  const int32_t* starts, int64_t batch, int32_t max_tree, const int32_t* block_table,
                                  int32_t max_blocks, const int32_t* seq_lens, int32_t window, int32_t sinks, void* out,
                                  int32_t ot, void* workspace, size_t ws_bytes, void* stream) {
  if (window < 0 || sinks < 0 || max_tree <= 0) return HQ_ERR_INVALID_ARG;
  if (max_tree > 64 || (window != 0 && window < max_tree)) return HQ_ERR_UNSUPPORTED;
  hq_cache_attn_args a;
  bool run;
  hq_status st = attention_args(kp, k, vp, v, q, qt, batch, rows, heads_q, scale, block_table, max_blocks, seq_lens, window,
                                sinks, out, ot, &a, &run);
  if (st != HQ_OK || !run) return st;
  if (!masks || !aligned(masks, 8) || !starts || !aligned(starts, 4)) return HQ_ERR_INVALID_ARG;
  const TreeSize s =
      tree_size(batch, rows, k->heads, a.group, (int64_t)max_blocks * k->block_tokens, max_tree, window, sinks);
  a.masks = masks;
  a.starts = starts;
  a.rows = (int32_t)rows;
  a.max_rows = max_tree;
  a.by_group = hq_divide_by((uint32_t)a.group);
  while (1 << a.tile_shift < s.tile) ++a.tile_shift;
  a.max_tiles = (int32_t)s.tiles;
  a.items = s.items;
  a.joins = s.joins;
  a.join = s.seen > HQ_CACHE_WHOLE;
  // workgroups of both launches
  if (s.items > kMaxGroups / k->heads ||
      s.joins * (((int64_t)max_tree * heads_q + 3) / 4) > kMaxGroups)
    return HQ_ERR_UNSUPPORTED;
  if (a.join && (!workspace || !aligned(workspace, 16) || ws_bytes < s.bytes)) return HQ_ERR_INVALID_ARG;
  if ((st = check_device(kp)) != HQ_OK || (st = check_device(vp)) != HQ_OK) return st;
  if (a.join) {
    a.part_acc = (float*)workspace;
    a.part_m = a.part_acc + s.parts * HQ_TILE;
    a.part_l = a.part_m + s.parts;
    a.parts = (hq_cache_of*)(a.part_l + s.parts);
    a.split = (int32_t*)(a.parts + batch);
  }
  return hip_status(hq_launch_cache_tree(a, k->format, stream));
}

}  // extern "C"
