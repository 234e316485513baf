"""The tree attention's partial sums lie inside its workspace, whichever row tile the rule takes for
a call's rows, drafted tokens of no sequence among them; on the CPU with a stand-in launcher."""
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23406_amd", "csrc")

# A line of a call's sizes in; its status, the workspace's bytes, the end of what its launch may
# write there, and the tile's rows out.
PROGRAM = r"""
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include "hq_internal.h"

static hq_cache_attn_args got;
extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
int hq_launch_rope_table(const hq_rope_table_args&, void*) { return 0; }
int hq_launch_rope(const hq_rope_args&, void*) { return 0; }
int hq_launch_cache_append(const hq_cache_append_args&, int, void*) { return 0; }
int hq_launch_cache_attention(const hq_cache_attn_args&, int, void*) { return 0; }
int hq_launch_cache_tree(const hq_cache_attn_args& a, int, void*) { got = a; return 0; }

int main() {
  alignas(16) static char some[64], *const ws = (char*)(1ull << 40);  // addresses alone
  long heads, group, batch, blocks, rows;
  int most, window, sinks;
  while (scanf("%ld %ld %ld %ld %ld %d %d %d", &heads, &group, &batch, &blocks, &rows, &most, &window, &sinks) == 8) {
    hq_plan_s p = {};
    p.tile = HQ_TILE;
    p.cols = heads * HQ_TILE;
    hq_cache k = {some, some, 8, 16, (int32_t)heads, HQ_INT8, 0, nullptr}, v = k;
    const int32_t hq = (int32_t)(heads * group);
    const size_t need = hq_cache_tree_workspace_bytes(&k, batch, hq, (int32_t)blocks, most, window, sinks);
    got = {};
    const int st = hq_cache_tree_attention(&p, &k, &p, &v, some, HQ_BF16, rows, hq, 0.1f, (const uint64_t*)some,
                                           (const int32_t*)some, batch, most, (const int32_t*)some, (int32_t)blocks,
                                           (const int32_t*)some, window, sinks, some, HQ_FP32, ws, need, nullptr);
    size_t end = 0;
    bool parts = true;
    if (st == HQ_OK && got.join) {
      end = (size_t)((char*)(got.split + got.joins + 1) - ws);
      // sums of every row of every item, before the maxima, these before the weights' sums
      const int64_t n = got.items * got.heads_kv << got.tile_shift;
      parts = got.part_m - got.part_acc >= n * HQ_TILE && got.part_l - got.part_m >= n && (float*)got.parts - got.part_l >= n;
    }
    printf("%d %zu %zu %d %d\n", st, need, end, 1 << got.tile_shift, (int)parts);
  }
}
"""


def test_partial_sums_lie_in_the_workspace(tmp_path):
    src, exe = tmp_path / "layout.cpp", tmp_path / "layout"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), "-o", str(exe), str(src),
                    *(os.path.join(CSRC, f) for f in ("hq_rope_host.cpp", "hq_cache_tree_host.cpp"))], check=True)
    r, cases = random.Random(4), []
    for _ in range(4000):
        heads, group, batch = r.choice([1, 2, 3, 8, 16, 64]), r.randint(1, 16), int(2 ** r.uniform(0, 9))
        blocks, most = int(2 ** r.uniform(0, 11)), r.randint(1, 64)
        rows = r.choice([1, batch, batch * most, batch * most * 3 // 4, batch * most + 1000, r.randint(1, batch * most)])
        cases.append((heads, group, batch, blocks, max(rows, 1), most, r.choice([0, 0, 64, 2000]), r.choice([0, 100])))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), check=True, capture_output=True,
                         text=True).stdout.split("\n")
    tiles = set()
    for c, line in zip(cases, out):
        st, need, end, tile, parts = map(int, line.split())
        assert st == 0 or (st == -2 and c[0] * c[1] * c[2] > 1 << 12), (c, line)
        assert end <= need and parts, (c, line)
        if end:
            tiles.add(tile)
    assert tiles == {16, 32, 128}
