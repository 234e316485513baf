"""Windowed and tree attention of so many sequences that none is split, in blocks of 16: a wave's way
is longer than the 64 blocks whose ids it asks for at once, and jumps over more than that between
sinks and window.  Against the definitions in 64 bits (tests/rows64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W

pytestmark = pytest.mark.gpu
N, B, HEADS, BT, MOST = R.N, 300, 2, 16, 5500
LOOKED_AT = [0, 1, 2, 150, 297, 298, 299]  # sequences that are compared


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def cache(hq, fmt, lens):
    kp, vp = R.plans(hq, HEADS)
    kc, vc = (R.random_cache(hq, p, fmt, 200, HEADS, BT, 10 * i + 3) for i, p in ((1, kp), (2, vp)))
    g = torch.Generator().manual_seed(33)
    table = torch.randint(0, 200, (len(lens), -(-MOST // BT)), generator=g).to(torch.int32)
    return kp, vp, kc, vc, table, g


def lengths():
    lens = np.full(B, 5000)
    lens[[1, 150, 298]] = [MOST, 17, 4999]
    return lens


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "mxfp4"])
@pytest.mark.parametrize("window,sinks", [(4700, 20), (4096, 1), (2000, 1500), (MOST, 0)])
def test_windows(hq, fmt, window, sinks):
    print(f"[long ways] window {fmt} {window} {sinks}", flush=True)
    lens = lengths()
    kp, vp, kc, vc, table, g = cache(hq, fmt, lens)
    q = torch.randn((B, HEADS, N), generator=g)
    out = hq.hq_cache_window_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), torch.from_numpy(lens).to(torch.int32).cuda(), window,
                                       sinks).cpu().numpy()
    kv, vv = R.values(kc), R.values(vc)
    for b in LOOKED_AT:
        want, tol = W.attend(q[b:b + 1].numpy(), kv, vv, table[b].numpy(), W.visible(int(lens[b]), window, sinks)[None], BT, N ** -0.5,
                             HEADS, 1)
        W.check(out[b:b + 1], want, tol)


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "mxfp4"])
@pytest.mark.parametrize("window,sinks,group,tree", [(0, 0, 1, 2), (4700, 20, 1, 2), (2000, 1500, 4, 7), (0, 0, 8, 16)])
def test_trees(hq, fmt, window, sinks, group, tree):
    print(f"[long ways] tree {fmt} {window} {sinks} {group} x {tree}", flush=True)
    lens, rng = lengths(), np.random.default_rng(4)
    kp, vp, kc, vc, table, g = cache(hq, fmt, lens)
    trees = np.full(B, tree)
    trees[2] = 0
    masks = [m for n in trees for m in W.random_tree(rng, int(n))]
    starts = np.concatenate(([0], np.cumsum(trees))).astype(np.int32)
    q = torch.randn((int(starts[-1]), HEADS * group, N), generator=g)
    out = hq.hq_cache_tree_attention(kp, kc, vp, vc, q.cuda(), W.mask_tensor(masks).cuda(), torch.from_numpy(starts).cuda(), tree,
                                     table.cuda(), torch.from_numpy(lens).to(torch.int32).cuda(), window=window, sinks=sinks).cpu().numpy()
    kv, vv = R.values(kc), R.values(vc)
    for b in LOOKED_AT:
        r = slice(starts[b], starts[b + 1])
        if trees[b] == 0:
            continue
        live = W.tree_visible(int(lens[b]), masks[r], window, sinks)
        want, tol = W.attend(q[r].numpy(), kv, vv, table[b].numpy(), live, BT, N ** -0.5, HEADS, group)
        W.check(out[r], want, tol, scale=N ** -0.5)
