"""What the host code of a cache attention hands to its launches, on the CPU with stand-in launchers:
which sequences the join reaches, and what is refused before anything is launched."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23406_amd", "csrc")

# A line of `batch heads group max_blocks` in, `status launched items joins` out.
PROGRAM = r"""
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include "hq_internal.h"

static hq_cache_attn_args seen;
static int launched;
extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
int hq_launch_cache_write(const hq_cache_io_args&, int, int, void*) { return 0; }
int hq_launch_cache_read(const hq_cache_io_args&, int, void*) { return 0; }
int hq_launch_norm_prep(const hq_norm_args&, void*) { return 0; }
int hq_launch_cache_attention(const hq_cache_attn_args& a, int, void*) { seen = a; ++launched; return 0; }

int main() {
  alignas(16) static char some[16];  // an address; nothing here reads behind one
  long batch, heads, group, blocks;
  while (scanf("%ld %ld %ld %ld", &batch, &heads, &group, &blocks) == 4) {
    hq_plan_s p = {};
    p.tile = HQ_TILE;
    p.cols = heads * HQ_TILE;
    hq_cache c = {some, some, 1, 16, (int32_t)heads, HQ_INT8, 0, nullptr};
    launched = 0;
    const int st = hq_cache_attention(&p, &c, &p, &c, some, HQ_FP32, batch, (int32_t)(heads * group), 0.1f, (int32_t*)some,
                                      (int32_t)blocks, (int32_t*)some, some, HQ_FP32, some, (size_t)1 << 62, nullptr);
    printf("%d %d %ld %ld\n", st, launched, launched ? (long)seen.items : 0, launched ? (long)seen.joins : 0);
  }
}
"""


@pytest.fixture(scope="module")
def attend(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("cache_launch")
    src, exe = tmp / "launch.cpp", tmp / "launch"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, "-o", str(exe),
                    str(src), os.path.join(CSRC, "hq_cache_host.cpp")], check=True, timeout=300)

    def calls(cases):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), check=True,
                             capture_output=True, text=True, timeout=60).stdout
        return [tuple(map(int, line.split())) for line in out.split("\n") if line]

    return calls


def test_the_join_reaches_every_split_sequence(attend):
    """Up to 64 sequences workgroup b of the join takes sequence b; of more, the b-th of those that are
    split.  Long sequences stand where the batch ends, in its middle, or everywhere."""
    shapes = [(b, h) for b in (1, 2, 16, 33, 34, 48, 57, 58, 63, 64, 65, 66, 200) for h in (1, 8, 9, 12, 16, 17, 32, 64, 300)]
    blocks = 512
    checked = 0
    for (batch, heads), (st, launched, items, joins) in zip(shapes, attend([(b, h, 1, blocks) for b, h in shapes])):
        assert st == 0 and launched == 1
        at = np.arange(batch)
        for lens in (np.where(at == batch - 1, 16 * blocks, 100), np.where(at == batch // 2, 16 * blocks, 0),
                     np.where(at >= batch - 2, 16 * blocks, 1), np.full(batch, 16 * blocks)):
            even = -(-int(lens.sum()) * heads // 512)
            for eighths in range(8, 17):  # the kernel takes one of these
                chunk = max(512, ((even * eighths >> 3) + 127) // 128 * 128)
                split = np.nonzero(-(-lens // chunk) > 1)[0]
                checked += len(split)
                assert len(split) <= joins, (batch, heads)
                if batch <= 64 and len(split):
                    assert split[-1] < joins, (batch, heads, split[-1], joins)
    assert checked > 1000


def test_the_join_fits_a_grid(attend):
    """2^24 workgroups of 256 are more threads than a grid holds.  From 512 KV heads on a chunk is at least
    all tokens together: nothing is split, and nothing joined."""
    shapes = [(b, h, g) for b in (1, 3, 4, 16, 63, 64, 65, 100) for g in (1, 16)
              for h in (1, 8, 64, 256, 511, 512, 513, 4096, 1 << 16, 1 << 18, 1 << 20)]
    done = 0
    for (batch, heads, group), (st, launched, items, joins) in zip(shapes, attend([s + (65,) for s in shapes])):
        if items_past_a_grid(batch, heads):
            assert st == -2 and not launched
            continue
        assert st == 0 and launched == 1, (batch, heads, group)
        assert joins * heads * group < 1 << 20, (batch, heads, group, joins)
        assert (joins == 0) == (heads >= 512)
        done += 1
    assert done > 100


def items_past_a_grid(batch, heads):
    return min(3 * batch, batch + 512 // heads + 1) * heads >= 1 << 24
