"""What the host code of rotary positions, the cache's append and the windowed and tree attentions
refuses, and what it hands to its launches, on the CPU with stand-in launchers."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23406_amd", "csrc")

# A line `name change` in, `name change status launches` out: a call that is right but for the change.
PROGRAM = r"""
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include <math.h>
#include <string>
#include "hq_internal.h"

static int launched, device;
extern "C" hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
int hq_launch_rope_table(const hq_rope_table_args&, void*) { return ++launched, 0; }
int hq_launch_rope(const hq_rope_args&, void*) { return ++launched, 0; }
int hq_launch_cache_append(const hq_cache_append_args&, int, void*) { return ++launched, 0; }
int hq_launch_cache_attention(const hq_cache_attn_args&, int, void*) { return ++launched, 0; }
int hq_launch_cache_tree(const hq_cache_attn_args&, int, void*) { return ++launched, 0; }

int main() {
  alignas(16) static char some[4096];  // addresses; nothing here reads behind one but the axes
  char name[64], change[64];
  while (scanf("%63s %63s", name, change) == 2) {
    const std::string call = name, c = change;
    device = c == "device";
    launched = 0;
    hq_plan_s p = {}, other;
    p.tile = HQ_TILE;
    p.cols = 512;
    other = p;
    if (c == "plan_tile") p.tile = 256;
    if (c == "plan_dither") p.dither = 1;
    if (c == "plan_cols") p.cols = 256;
    hq_cache k = {some, some + 16, 8, 64, 4, HQ_INT8, 0, nullptr}, v = {some + 32, some + 48, 8, 64, 4, HQ_INT8, 0, nullptr};
    if (c == "block_tokens") k.block_tokens = v.block_tokens = 24;
    if (c == "formats") v.format = HQ_E4M3;
    if (c == "heads") v.heads = 2;
    if (c == "format") k.format = v.format = HQ_BF16;
    if (c == "shared") v.codes = k.codes;
    uint8_t axis[64] = {};
    for (int i = 0; i < 64; ++i) axis[i] = i % 3;
    hq_rotary r = {(const float*)some, 100, 128, 0, 3, 0, axis, nullptr};
    if (c == "dims_odd") r.dims = 33;
    if (c == "dims_0") r.dims = 0;
    if (c == "dims_130") r.dims = 144;
    if (c == "dims_24") r.dims = 24;
    if (c == "axes_0") r.axes = 0;
    if (c == "axes_5") r.axes = 5;
    if (c == "axis_past") r.axes = 2;
    if (c == "axis_null") r.axis = nullptr;
    if (c == "one_axis_null") r.axis = nullptr, r.axes = 1;
    if (c == "positions_0") r.positions = 0;
    if (c == "positions_many") r.positions = 1ll << 31;
    if (c == "interleaved_2") r.interleaved = 2;
    if (c == "table_null") r.table = nullptr;
    if (c == "table_off") r.table = (const float*)(some + 4);
    const hq_rotary* rp = c == "rope_null" ? nullptr : &r;
    const int32_t* pos = c == "pos_null" ? nullptr : (const int32_t*)(some + (c == "pos_off" ? 2 : 0));
    const int64_t rows = c == "rows_0" ? 0 : c == "rows_neg" ? -1 : c == "rows_many" ? 1 << 27 : 10;
    const int32_t xt = c == "type" ? HQ_INT8 : HQ_BF16;
    const int64_t ld = c == "ld_short" ? 504 : c == "ld_odd" ? 513 : 512;
    const void* x = c == "x_null" ? nullptr : some + (c == "x_off" ? 8 : 64);
    void* y = c == "y_null" ? nullptr : some + (c == "y_off" ? 8 : 128);
    int st = -100;
    if (call == "table")
      st = hq_rope_table((const double*)(c == "x_null" ? nullptr : some), c == "pairs_0" ? 0 : c == "pairs_65" ? 65 : 64,
                         c == "rows_0" ? 0 : c == "rows_neg" ? -1 : c == "positions_many" ? 1ll << 31 : 10,
                         c == "factor" ? INFINITY : 1.0f, (float*)y, nullptr);
    if (call == "rope")
      st = hq_rope(rp, x, xt, ld, rows, c == "heads_0" ? 0 : 4, pos, c == "transposed_2" ? 2 : 0,
                   c.substr(0, 8) == "in_place" ? (void*)x : y, c == "out_type" ? HQ_MXFP4 : c == "in_place_type" ? HQ_FP32 : HQ_BF16,
                   c == "in_place_ld" ? 520 : 512, nullptr);
    if (call == "append") {
      const bool keys = c == "keys", none = c == "no_queries";
      st = hq_cache_append(c == "plan_null" ? nullptr : &p, x, ld, c == "cache_null" ? nullptr : &k, keys ? nullptr : &other,
                           keys || c == "v_null" ? nullptr : c == "v_off" ? some + 8 : some + 256, 512, keys ? nullptr : &v, xt, rows,
                           c == "slots_null" ? nullptr : (const int64_t*)(some + (c == "slots_off" ? 4 : 0)), rp, pos,
                           none || c == "q_null" ? nullptr : some + 512, c == "q_ld" ? 1016 : 1024, none || c == "q_heads" ? 0 : 8,
                           none || c == "q_out_null" ? nullptr : c.substr(0, 8) == "in_place" ? some + 512 : some + 1024,
                           c == "q_type" ? 7 : c == "in_place_type" ? HQ_FP32 : HQ_BF16, c == "in_place_ld" ? 1032 : 1024, nullptr);
    }
    const bool tree = call == "tree";
    if (tree || call == "window") {
      const int64_t batch = c == "batch_0" ? 0 : c == "batch_neg" ? -1 : 3;
      const int32_t hq = c == "heads_q" ? 6 : c == "group" ? 68 : c == "heads_q_0" ? 0 : 16;
      const int32_t blocks = c == "max_blocks_0" ? 0 : c == "long" ? 1 << 25 : 40;
      const int32_t window = c == "window_0" ? 0 : c == "window_neg" ? -1 : c == "window_small" ? 10 : c == "window_short" ? 512 : 2000;
      const int32_t sinks = c == "sinks_neg" ? -1 : c == "sinks" ? 5 : 0, most = c == "tree_0" ? 0 : c == "tree_65" ? 65 : 20;
      const float scale = c == "scale" ? NAN : 0.1f;
      const int32_t* table = c == "block_table_null" ? nullptr : (const int32_t*)some;
      const int32_t* lens = c == "lens_null" ? nullptr : (const int32_t*)some;
      const size_t need = tree ? hq_cache_tree_workspace_bytes(&k, 3, hq, blocks, most, window, sinks)
                               : hq_cache_window_workspace_bytes(&k, 3, hq, blocks, window, sinks);
      void* ws = c == "workspace_null" || c == "window_short" ? nullptr : some + (c == "workspace_off" ? 8 : 0);
      const size_t have = c == "workspace_small" ? need - 1 : need;
      const int32_t ot = c == "out_type" ? HQ_INT8 : HQ_FP32;
      if (tree)
        st = hq_cache_tree_attention(&p, &k, &other, &v, x, xt, rows, hq, scale, (const uint64_t*)(c == "masks_null" ? nullptr : some + (c == "masks_off" ? 4 : 0)),
                                     (const int32_t*)(c == "starts_null" ? nullptr : some), batch, most, table, blocks, lens, window,
                                     sinks, y, ot, ws, have, nullptr);
      else
        st = hq_cache_window_attention(&p, &k, &other, &v, x, xt, batch, hq, scale, table, blocks, lens, window, sinks, y, ot, ws,
                                       have, nullptr);
    }
    printf("%s %s %d %d\n", name, change, st, launched);
  }
}
"""

OK, INVALID, UNSUPPORTED = 0, -1, -2
ROTARY = {"dims_odd": INVALID, "dims_0": INVALID, "dims_130": INVALID, "dims_24": UNSUPPORTED, "axes_0": INVALID, "axes_5": INVALID,
          "axis_past": INVALID, "axis_null": INVALID, "one_axis_null": OK, "positions_0": INVALID, "positions_many": UNSUPPORTED,
          "interleaved_2": INVALID, "table_null": INVALID, "table_off": INVALID, "rope_null": INVALID, "pos_null": INVALID,
          "pos_off": INVALID}
ROWS = {"rows_0": OK, "rows_neg": INVALID, "rows_many": UNSUPPORTED, "type": INVALID, "ld_short": INVALID, "ld_odd": INVALID,
        "x_null": INVALID, "x_off": INVALID}
CACHES = {"plan_tile": UNSUPPORTED, "plan_dither": UNSUPPORTED, "plan_cols": INVALID, "block_tokens": UNSUPPORTED, "formats": INVALID,
          "heads": INVALID, "format": INVALID, "device": INVALID}
ATTENTION = {**CACHES, "type": INVALID, "out_type": INVALID, "x_null": INVALID, "x_off": INVALID, "y_null": INVALID, "y_off": INVALID,
             "batch_0": OK, "batch_neg": INVALID, "heads_q": INVALID, "heads_q_0": INVALID, "group": UNSUPPORTED,
             "max_blocks_0": INVALID, "long": UNSUPPORTED, "window_neg": INVALID, "sinks_neg": INVALID, "sinks": OK, "scale": INVALID,
             "block_table_null": INVALID, "lens_null": INVALID, "workspace_null": INVALID, "workspace_off": INVALID,
             "workspace_small": INVALID, "window_short": OK}
CASES = {
    "table": {"right": OK, "x_null": INVALID, "y_null": INVALID, "y_off": INVALID, "pairs_0": INVALID, "pairs_65": UNSUPPORTED,
              "rows_0": OK, "rows_neg": INVALID, "positions_many": UNSUPPORTED, "factor": INVALID},
    "rope": {"right": OK, **ROTARY, **ROWS, "heads_0": INVALID, "transposed_2": INVALID, "y_null": INVALID, "y_off": INVALID,
             "out_type": INVALID, "in_place": OK, "in_place_type": INVALID, "in_place_ld": INVALID},
    "append": {"right": OK, **ROTARY, **ROWS, **CACHES, "shared": INVALID, "keys": OK, "no_queries": OK, "plan_null": INVALID,
               "cache_null": INVALID, "v_null": INVALID, "v_off": INVALID, "slots_null": INVALID, "slots_off": INVALID,
               "q_null": INVALID, "q_ld": INVALID, "q_heads": INVALID, "q_out_null": INVALID, "q_type": INVALID, "in_place": OK,
               "in_place_type": INVALID, "in_place_ld": INVALID},
    "window": {"right": OK, **ATTENTION, "window_0": INVALID, "window_small": OK},
    "tree": {"right": OK, **ATTENTION, "rows_0": OK, "rows_neg": INVALID, "window_0": OK, "window_small": UNSUPPORTED, "tree_0": INVALID,
             "tree_65": UNSUPPORTED, "masks_null": INVALID, "masks_off": INVALID, "starts_null": INVALID},
}


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("rope_tree_launch")
    src, exe = tmp / "launch.cpp", tmp / "launch"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, "-o", str(exe), str(src),
                    os.path.join(CSRC, "hq_rope_host.cpp"), os.path.join(CSRC, "hq_cache_tree_host.cpp")], check=True, timeout=300)
    asked = "".join(f"{name} {change}\n" for name, changes in CASES.items() for change in changes)
    out = subprocess.run([str(exe)], input=asked, check=True, capture_output=True, text=True, timeout=60).stdout
    return {(a, b): (int(st), int(n)) for a, b, st, n in (line.split() for line in out.split("\n") if line)}


@pytest.mark.parametrize("name", CASES)
def test_refusals(answers, name):
    """A right call launches once; a refused one, or one with nothing to do, nothing."""
    for change, want in CASES[name].items():
        st, launches = answers[name, change]
        nothing = change in ("rows_0", "batch_0")
        assert (st, launches) == (want, 1 if want == OK and not nothing else 0), (name, change)


def test_workspaces_serve_smaller_calls():
    """The tree's workspace never falls as a call grows, whichever row tile its rule takes."""
    from paper_2606_23406_amd import build, hq
    if not os.path.exists(build.LIB):
        build.build()
    L, r = hq.lib(), random.Random(1)

    def size(heads, batch, heads_q, blocks, tree, window, sinks):
        c = hq.CacheStruct(None, None, 8, 16, heads, 3, 0, None)
        return L.hq_cache_tree_workspace_bytes(C.byref(c), batch, heads_q, blocks, tree, window, sinks)

    for _ in range(20000):
        h, g, b = r.choice([1, 2, 3, 4, 8, 16, 64, 600]), r.randint(1, 16), int(2 ** r.uniform(0, 11))
        nb, t, w, s = int(2 ** r.uniform(0, 11)), r.randint(1, 64), r.choice([0, 64, 100, 3000]), r.choice([0, 5, 300])
        more = (h, b + r.choice([0, 1, 3, 100]), h * r.randint(g, 16), nb + r.choice([0, 1, 50]), r.randint(t, 64),
                0 if w == 0 or r.random() < 0.3 else w + r.randint(0, 500), s + r.randint(0, 50))
        assert size(*more) >= size(h, b, h * g, nb, t, w, s), (h, g, b, nb, t, w, s, more)


CHUNKS = r"""
#include <stdio.h>
#include "hq_internal.h"
int main() {
  long batch, heads, seen, tiles;
  while (scanf("%ld %ld %ld %ld", &batch, &heads, &seen, &tiles) == 4)
    printf("%ld %ld\n", (long)hq_tree_items(batch, heads, seen, tiles), (long)hq_cache_joins(batch, heads));
}
"""


def test_chunks_of_trees_fit_the_grid(tmp_path):
    """The chunks that the kernels cut trees into (their arithmetic, here in Python), once for each of a
    tree's row tiles, are never more than the bound that the grid and the workspace go by."""
    src, exe = tmp_path / "chunks.cpp", tmp_path / "chunks"
    src.write_text(CHUNKS)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    r, cases = random.Random(2), []
    for _ in range(300):
        batch, heads, most = int(2 ** r.uniform(0, 10)), r.choice([1, 2, 3, 8, 16, 64, 600]), int(2 ** r.uniform(10.1, 15))
        tiles = r.choice([1, 2, 3, 8, 32])
        cases.append((batch, heads, most, tiles))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), check=True, capture_output=True, text=True).stdout
    for (batch, heads, most, tiles), line in zip(cases, out.split("\n")):
        items, joins = map(int, line.split())
        for lens in ([most] * batch, [r.randint(0, most) for _ in range(batch)], [most] + [1] * (batch - 1)):
            of = [r.randint(1, tiles) for _ in lens]
            even = -(-sum(n * t for n, t in zip(lens, of)) * heads // 512)
            for eighths in range(8, 17):
                chunk = max(512, ((even * eighths >> 3) + 127) // 128 * 128)
                parts = [max(1, -(-n // chunk)) for n in lens]
                assert sum(p * t for p, t in zip(parts, of)) <= items
                assert sum(p > 1 for p in parts) <= joins
