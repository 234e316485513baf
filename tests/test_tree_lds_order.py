"""A wave's lanes hand values to each other through LDS in the tree attention: in the compiler's
optimized form of the kernels a fence stands between every write to LDS and the reads behind it in
its basic block, so that no later pass may move a read above the write that it depends on."""
import os
import re
import subprocess

import pytest

from paper_2606_23406_amd import build

SRC = os.path.join(build.CSRC, "hq_cache_tree.hip")
WRITE = re.compile(r"\bstore .*ptr addrspace\(3\)")
READ = re.compile(r"= load .*ptr addrspace\(3\)")
FENCE = re.compile(r'\bfence syncscope\("(wavefront|workgroup)"\) (acquire|release)')


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("tree_ir") / "tree.ll"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-S", "-emit-llvm", "--offload-device-only", "-o", str(out), SRC], check=True,
                   capture_output=True, timeout=600)
    return dict(re.findall(r"define amdgpu_kernel void @\w*?\d+(hq_cache_tree_kernel\w+?)EEEv\S*\((.*?)\n}\n", out.read_text(), re.S))


def test_writes_to_lds_are_fenced_from_the_reads_behind_them(kernels):
    """Kernels of 16 and 32 rows: int8, E4M3 and MXFP4, four and eight waves.  (MXFP4's tokens' scales
    are written and read within a step.)"""
    assert len(kernels) == 9
    for name, body in kernels.items():
        pending, fences = None, set()
        writes = 0
        for line in body.split("\n"):
            if re.match(r"\d+:", line):  # another basic block, which need not run behind the one above
                pending = None
            elif WRITE.search(line):
                pending, fences = line, set()
                writes += 1
            elif m := FENCE.search(line):
                fences.add(m.group(2))
            elif READ.search(line):
                assert pending is None or fences == {"acquire", "release"}, (name, pending.strip(), line.strip())
                pending = None
        assert writes > 10, name
