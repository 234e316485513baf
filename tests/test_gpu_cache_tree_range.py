"""The tree attention at both ends of fp32's range, in tiles of 16, 32 and 128 rows, against the
definitions in 64 bits (tests/rows64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W
from tests.test_gpu_cache_tree import FMTS, Case, hq  # noqa: F401  (hq: the fixture)
from tests.test_gpu_cache_tree_full_tiles import FILL, MOST, Full

pytestmark = pytest.mark.gpu
U = R.U
TILES = ["16", "32", "128"]


def case(hq, fmt, tile, lens, trees, **kw):
    """A few sequences in one of the row tiles."""
    heads, group, bt, pool = 2, 4, 32, kw.pop("pool", 60)
    if tile == "16":
        return Case(hq, fmt, lens, [min(t, 4) for t in trees], heads, group, bt, pool=pool, max_tree=4, **kw)
    if tile == "32":
        lens, trees = list(lens) + [3] * FILL, [min(t, 12) for t in trees] + [1] * FILL
        return Case(hq, fmt, lens, trees, heads, group, bt, pool=pool, max_tree=12, **kw)
    return Full(hq, fmt, list(lens) + [3] * FILL, list(trees) + [1] * FILL, heads, group, bt, pool=pool, max_tree=MOST, **kw)


def set_scales(c, cache, exponents):
    """Value or key scales 2^exponents, [blocks, block_tokens]."""
    e = exponents[:, None, :].expand(cache.scales.shape[:3])
    if R.name(cache) == "mxfp4":
        cache.scales.copy_((e + 127).to(torch.uint8)[..., None].expand(cache.scales.shape))
    else:
        cache.scales.copy_(torch.ldexp(torch.ones(()), e))


def compare(c, out):
    """Each row within its bound, which goes by the largest value that it sees; the rows together, too."""
    ref, tol = c.reference()
    off = np.abs(out.cpu().numpy().astype(np.float64) - ref)
    assert np.isfinite(ref).all() and (off <= tol).all(), float((off / tol).max())  # a NaN is not
    size = np.linalg.norm(ref, axis=-1)
    assert (np.linalg.norm(off, axis=-1) <= 64 * U * 4 * size + 1e-30).all()
    assert torch.equal(c.run(), out) and c.kc.read_stats()["status"] == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("exponent", [38, 90])
def test_zero_vectors_beside_large_values(hq, fmt, tile, exponent):
    """Half of the tokens are zero vectors, whole steps of them: they keep their part of the weights."""
    print(f"[tree] range zeros {fmt} {tile} {exponent}", flush=True)
    c = case(hq, fmt, tile, [400, 90, 1500], [9, 20, 30], seed=42)
    set_scales(c, c.vc, torch.full((60, 32), exponent))
    c.vc.codes[::2] = 0
    c.vc.scales[::2] = 0
    compare(c, c.run())
