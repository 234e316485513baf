"""Trees over a window: table entries of blocks that no row can look at are not used."""
import pytest
import torch

from tests.test_gpu_cache_tree import FMTS, Case, hq  # noqa: F401  (hq: the fixture)
from tests.test_gpu_cache_tree_full_tiles import FILL, MOST, Full

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", [16, 32, 128])
@pytest.mark.parametrize("window,sinks", [(64, 0), (64, 1), (65, 17), (80, 32), (100, 16), (333, 5)])
def test_freed_blocks(hq, fmt, tile, window, sinks):
    """Every entry that the header allows to be freed is no block at all: the same bits, and no report."""
    print(f"[tree] freed {fmt} {tile} {window} {sinks}", flush=True)
    lens, trees, bt = [600, 1499, 77, 160, 97], [5, 30, 13, 1, 16], 16
    if tile == 16:
        c = Case(hq, fmt, lens, [min(t, 4) for t in trees], 2, 4, bt, pool=60, max_tree=4, window=window, sinks=sinks)
    else:
        of, most = (Case, 12) if tile == 32 else (Full, MOST)
        c = of(hq, fmt, lens + [3] * FILL, [min(t, most) for t in trees] + [1] * FILL, 2, 4, bt, pool=60, max_tree=most,
               window=window, sinks=sinks)
    want, freed = c.check(), 0
    for b, (n, tree) in enumerate(zip(c.lens, c.trees)):
        for i in range(c.table.shape[1]):
            if (i + 1) * bt <= n - tree - window and i * bt >= sinks or i * bt >= n:
                c.table[b, i] = [-1, 60, -2 ** 31, 2 ** 31 - 1][i % 4]
                freed += i * bt < n
    assert freed > 40
    assert torch.equal(c.run(), want) and c.kc.read_stats()["status"] == 0
