"""The tree attention in tiles of 128 rows, which a call takes where its rows fill them: rows of no
sequence behind the last one make the small sequences of these tests such calls (against
tests/rows64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W
from tests.test_gpu_cache_tree import FMTS, Case, hq  # noqa: F401  (hq: the fixture)

pytestmark = pytest.mark.gpu
MOST, FILL = 30, 300  # drafted tokens of a sequence at most, sequences of three tokens with one of them


class Full(Case):
    """A call with as many rows as all of its sequences could have."""

    def run(self, **kw):
        rows, full = self.q.shape[0], len(self.lens) * self.max_tree
        q, masks, out = self.q, self.masks, kw.pop("out", None)
        self.q = torch.cat([q, torch.full((full - rows, *q.shape[1:]), float("nan"), dtype=q.dtype)])
        self.masks = list(masks) + [(1 << 64) - 1] * (full - rows)
        try:
            if out is not None:
                kw["out"] = torch.full(self.q.shape, 7.0, dtype=out.dtype, device="cuda")
            got = super().run(**kw)
        finally:
            self.q, self.masks = q, masks
        assert (got[rows:] == (0.0 if out is None else 7.0)).all()  # left as they were
        return got[:rows]


def case(hq, fmt, lens, trees, **kw):
    if kw.get("masks") is not None:
        kw["masks"] = kw["masks"] + [1] * FILL
    return Full(hq, fmt, list(lens) + [3] * FILL, list(trees) + [1] * FILL, kw.pop("heads", 2), 4, kw.pop("bt", 32),
                pool=kw.pop("pool", 60), max_tree=MOST, **kw)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("lens,trees", [([0, 1, 2, 15, 16, 17, 33, 64, 65, 100, 129, 511], [0, 1, 2, 9, 16, 1, 30, 30, 5, 12, 13, 29]),
                                        ([3000, 1025, 40, 1024, 513], [30, 17, 30, 4, 8])])
def test_lengths(hq, fmt, lens, trees):
    print(f"[tree] full tiles {fmt} {max(lens)}", flush=True)
    case(hq, fmt, lens, trees).check()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(64, 0), (70, 17), (100, 300), (900, 5)])
def test_windows(hq, fmt, window, sinks):
    print(f"[tree] full tiles windows {fmt} {window} {sinks}", flush=True)
    case(hq, fmt, [300, 64, 65, 80, 513, 1, 0, 2000], [20, 30, 1, 30, 30, 1, 0, 28], window=window, sinks=sinks, seed=4).check()


@pytest.mark.parametrize("spread", [3, 10])
def test_scales_far_apart(hq, spread):
    c = case(hq, "int8", [400, 90, 1500], [9, 20, 30], seed=12)
    g = torch.Generator().manual_seed(1)
    c.vc.scales.copy_(10.0 ** (spread * (2 * torch.rand(c.vc.scales.shape, generator=g) - 1)))
    c.vc.scales[:, :, 5::11] = 0.0
    c.kc.scales[:, :, 7::13] = 0.0
    ref, tol = c.reference()
    off = np.abs(c.run().cpu().numpy() - ref)
    assert (off <= tol).all()
    assert (np.linalg.norm(off, axis=-1) <= 64 * R.U * 4 * np.linalg.norm(ref, axis=-1) + 1e-30).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("side", ["k", "v"])
def test_tokens_that_are_not_finite(hq, fmt, side):
    """One drafted token is NaN: the rows that see it, and no others; stale codes of any bits behind the
    sequence and in a block that the cache does not have."""
    n = MOST
    masks = [1, 2, 5] + [(1 << i) | 1 for i in range(3, n)]  # token 1 is a leaf
    c = case(hq, fmt, [200], [n], masks=masks, seed=11, pool=None, window=64, sinks=3)
    clean = c.check().cpu().numpy()
    cache = c.kc if side == "k" else c.vc
    for t in (200 - n + 1, 50):
        blk = int(c.table[0, t // 32])
        cache.codes[blk, :, t % 32] = 0
        cache.scales[blk, :, t % 32] = float("nan") if fmt != "mxfp4" else 255
    for x in (c.kc, c.vc):
        blk = int(c.table[0, 6])
        x.codes.view(torch.uint8)[blk, :, 8:] = 0x7F if fmt == "e4m3" else 0x80
        x.scales[blk, :, 8:] = float("nan") if fmt != "mxfp4" else 255
    out = c.run().cpu().numpy()
    assert np.isnan(out[1]).all() and not np.isnan(np.delete(out, 1, 0)).any()
    assert np.array_equal(np.delete(out, 1, 0), np.delete(clean, 1, 0))


def test_bad_blocks(hq):
    c = case(hq, "e4m3", [100, 70, 1300, 40], [5, 9, 30, 8], seed=9)
    c.table[0, 1], c.table[1, 0], c.table[2, 7], c.table[3, :] = c.kc.blocks, -1, 1 << 30, -5
    W.check(c.run().cpu().numpy(), *c.reference())
    assert c.kc.read_stats()["status"] == -1 & 0xFFFFFFFF


@pytest.mark.parametrize("heads,group", [(1, 16), (3, 5), (5, 7), (8, 4)])
def test_heads(hq, heads, group):
    """Head layouts whose rows end inside a tile."""
    rows, fill = min(64, 120 // group), 600
    print(f"[tree] full tiles heads {heads} x {group} x {rows}", flush=True)
    Full(hq, "int8", [301, 64, 130] + [3] * fill, [rows, min(rows, 30), max(1, rows // 2)] + [1] * fill, heads, group, 32, seed=heads,
         qdt=torch.bfloat16, pool=40, max_tree=rows).check()


@pytest.mark.parametrize("factor", [1e-30, 1e-6, 1e6, 1e20])
def test_queries_and_values_of_any_size(hq, factor):
    c = case(hq, "e4m3", [300, 40, 1100], [9, 30, 20], seed=13)
    c.q = c.q * factor
    c.kc.scales.copy_(c.kc.scales / factor)
    W.check(c.run().cpu().numpy(), *c.reference())
    c.vc.scales.copy_(c.vc.scales * factor)
    W.check(c.run().cpu().numpy(), *c.reference())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("group,trees", [(4, [64, 63, 50, 64]), (8, [32, 31, 16, 20]), (16, [24, 8, 7, 64])])
def test_split_sequences(hq, fmt, group, trees):
    """Several tiles of a sequence, and chunks that are joined."""
    most = max(trees)
    print(f"[tree] full tiles split {fmt} {group} x {most}", flush=True)
    Full(hq, fmt, [4000, 2500, 1030, 700] + [40] * 12, trees + [most] * 12 if most < 40 else trees + [40] * 12, 8, group, 48, seed=14,
         pool=50, max_tree=most).check()
