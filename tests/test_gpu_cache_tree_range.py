"""The tree attention at both ends of fp32's range, in tiles of 16, 32 and 128 rows, against the
definitions in 64 bits (tests/rows64.py): value scales of any size, zero vectors among them,
and scores of any size."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W
from tests import test_gpu_cache_long_ways as L
from tests.test_gpu_cache_tree import FMTS, Case, hq  # noqa: F401  (hq: the fixture)
from tests.test_gpu_cache_tree_full_tiles import FILL, MOST, Full

pytestmark = pytest.mark.gpu
N, U = R.N, R.U
TILES = ["16", "32", "128"]
TOP = {"int8": 127.0, "e4m3": 448.0, "mxfp4": 6.0}


def case(hq, fmt, tile, lens, trees, **kw):
    """A few sequences in one of the row tiles."""
    heads, group, bt, pool = 2, 4, 32, kw.pop("pool", 60)
    if tile == "16":
        return Case(hq, fmt, lens, [min(t, 4) for t in trees], heads, group, bt, pool=pool, max_tree=4, **kw)
    if tile == "32":
        lens, trees = list(lens) + [3] * FILL, [min(t, 12) for t in trees] + [1] * FILL
        return Case(hq, fmt, lens, trees, heads, group, bt, pool=pool, max_tree=12, **kw)
    return Full(hq, fmt, list(lens) + [3] * FILL, list(trees) + [1] * FILL, heads, group, bt, pool=pool, max_tree=MOST, **kw)


def set_scales(cache, exponents):
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


# the largest scale's exponent whose vectors, as random_cache draws them, stay below 3.4e38
LARGEST = {"int8": 120, "e4m3": 119, "mxfp4": 124}


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("low,high", [(95, 108), (110, None), (-40, None), (-120, -100), (-100, -20), (-90, 30)])
def test_value_scales(hq, fmt, tile, low, high):
    """All scales large, all small, or from small to large; a score's weight does not depend on them."""
    print(f"[tree] range {fmt} {tile} {low} .. {high}", flush=True)
    c = case(hq, fmt, tile, [400, 90, 1500], [9, 20, 30], seed=40)
    c.vc.codes.copy_(R.random_cache(hq, c.vp, fmt, c.vc.blocks, 2, 32, 41).codes.cpu())
    g = torch.Generator().manual_seed(low + 200)
    set_scales(c.vc, torch.randint(low, LARGEST[fmt] + 1 if high is None else high, (60, 32), generator=g))
    compare(c, c.run())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("exponent", [38, 90, 118])
def test_zero_vectors_beside_large_values(hq, fmt, tile, exponent):
    """Half of the tokens are zero vectors, whole steps of them: they keep their part of the weights."""
    print(f"[tree] range zeros {fmt} {tile} {exponent}", flush=True)
    c = case(hq, fmt, tile, [400, 90, 1500], [9, 20, 30], seed=42)
    set_scales(c.vc, torch.full((60, 32), exponent))
    c.vc.codes[::2] = 0
    c.vc.scales[::2] = 0
    compare(c, c.run())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("exponent", [0, 100, 112, 118])
def test_many_tokens_of_small_weight(hq, fmt, tile, exponent):
    """One token has the largest weight, each of 16000 others 2^-17 of it: an eighth in all."""
    print(f"[tree] range weights {fmt} {tile} {exponent}", flush=True)
    c = case(hq, fmt, tile, [16000], [4], seed=43, pool=500)
    c.table[0] = torch.randperm(500, generator=torch.Generator().manual_seed(2))
    code = {"int8": 64, "e4m3": 0x38, "mxfp4": 0x22}[fmt]  # 64, 1 and 1
    unit = {"int8": 64.0, "e4m3": 1.0, "mxfp4": 1.0}[fmt]
    # queries whose transform is 128 in the first value alone, keys of one code: scores go by the key's scale
    c.kc.codes.copy_(torch.full(c.kc.codes.shape, code, dtype=c.kc.codes.dtype))
    d = torch.from_numpy(R.signs(R.SEED_K, 2 * N)).float().view(2, 1, N).expand(2, 4, N).reshape(1, 8, N)
    c.q = d.expand(c.q.shape).contiguous()
    # 17 bits: scale * 128 * unit * (2^0 - 2^-20 of the key) / 128 = 17 ln 2, nearly
    c.scale = 17 * np.log(2.0) / unit
    set_scales(c.kc, torch.full((c.kc.blocks, 32), -20))
    blk, at = int(c.table[0, 40]), 7
    c.kc.scales[blk, :, at] = 1.0 if fmt != "mxfp4" else 127
    set_scales(c.vc, torch.full((c.vc.blocks, 32), exponent))
    out = c.run()
    ref, _ = c.reference()
    # 16000 tokens: sums of the weights and of the products, and 60 roundings more; scores of 17 bits move a weight by 2 * 150 U * 17
    big = 2.0 ** exponent * TOP[fmt]
    rows = slice(0, 4)
    assert (np.abs(out[rows].cpu().numpy() - ref[rows]) <= (16060 + 2 * 150 * 17) * U * big).all()
    assert np.linalg.norm(out[rows].cpu().numpy() - ref[rows]) <= 64 * U * 17 * np.linalg.norm(ref[rows])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks,group,tree", [(0, 0, 1, 2), (2000, 1500, 4, 7), (0, 0, 8, 16)])
def test_large_values_on_long_ways(hq, fmt, window, sinks, group, tree):
    """Ways of more blocks than a wave asks for at once, gone over twice; the largest scales come late."""
    print(f"[tree] range long ways {fmt} {window} {sinks} {group} x {tree}", flush=True)
    lens = L.lengths()
    kp, vp, kc, vc, table, g = L.cache(hq, fmt, lens)
    exponents = torch.randint(-10, 90, (200, L.BT), generator=g)
    exponents[150:] += 25
    table[:, :-150] %= 150
    set_scales(vc, exponents)
    trees = np.full(L.B, tree)
    masks = [m for n in trees for m in W.random_tree(np.random.default_rng(5), int(n))]
    starts = np.concatenate(([0], np.cumsum(trees))).astype(np.int32)
    q = torch.randn((int(starts[-1]), L.HEADS * group, N), generator=g)
    out = hq.hq_cache_tree_attention(kp, kc, vp, vc, q.cuda(), W.mask_tensor(masks).cuda(), torch.from_numpy(starts).cuda(), tree,
                                     table.cuda(), torch.from_numpy(lens).to(torch.int32).cuda(), window=window, sinks=sinks).cpu().numpy()
    kv, vv = R.values(kc), R.values(vc)
    for b in L.LOOKED_AT:
        r = slice(starts[b], starts[b + 1])
        live = W.tree_visible(int(lens[b]), masks[r], window, sinks)
        want, tol = W.attend(q[r].numpy(), kv, vv, table[b].numpy(), live, L.BT, N ** -0.5, L.HEADS, group)
        W.check(out[r], want, tol, scale=N ** -0.5)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("exponent", [-9, 40, 70])
@pytest.mark.parametrize("size", [3e8, 1e30, -1e12])
def test_scores_of_any_size(hq, fmt, tile, exponent, size):
    """Every third token has the same largest score, exactly; the others are half of it below: the
    result is the mean of those tokens' values."""
    print(f"[tree] range scores {fmt} {tile} 2^{exponent} {size}", flush=True)
    c = case(hq, fmt, tile, [400, 90, 1500], [9, 20, 30], seed=44)
    code = {"int8": 64, "e4m3": 0x38, "mxfp4": 0x22}[fmt]
    unit = {"int8": 64.0, "e4m3": 1.0, "mxfp4": 1.0}[fmt]
    c.kc.codes.copy_(torch.full(c.kc.codes.shape, code, dtype=c.kc.codes.dtype))
    d = torch.from_numpy(R.signs(R.SEED_K, 2 * N)).float().view(2, 1, N).expand(2, 4, N).reshape(1, 8, N)
    c.q = d.expand(c.q.shape).contiguous()
    c.scale = abs(size) / unit  # of a key of scale 1
    top = torch.arange(32).expand(60, 32) % 3 == 1
    # scores size and size / 2, or -size / 2 and -size: every row sees a token before the tree
    if size < 0:
        c.q = -c.q
        set_scales(c.kc, torch.where(top, -1, 0))
    else:
        set_scales(c.kc, torch.where(top, 0, -1))
    c.vc.codes.copy_(R.random_cache(hq, c.vp, fmt, c.vc.blocks, 2, 32, 45).codes.cpu())
    set_scales(c.vc, exponent + torch.randint(-3, 4, (60, 32), generator=torch.Generator().manual_seed(1)))
    out = c.run().cpu().numpy()
    vv = R.values(c.vc)
    for b, n in enumerate(c.lens[:3]):
        r = range(c.starts[b], c.starts[b + 1])
        live = W.tree_visible(n, c.masks[r.start:r.stop])
        t = np.arange(n)
        blk = c.table[b].numpy()[t // 32]
        for i, row in enumerate(r):
            at = live[i] & (t % 32 % 3 == 1)
            mean = vv[blk[at], :, t[at] % 32].mean(0)  # [heads, 128]
            want = np.repeat((mean @ R.hadamard()) / N * R.signs(R.SEED_V, 2 * N).reshape(2, N), 4, 0)
            # weights are alike; their sum, the products' and the transform: (tokens + 60) U of the largest value
            big = np.sqrt((vv[blk[at], :, t[at] % 32] ** 2).sum(-1).max() / N)
            assert (np.abs(out[row] - want) <= (at.sum() + 60) * U * big).all(), (b, i)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("exponent", [-9, 60, 110])
def test_scores_far_below_before_others(hq, fmt, tile, exponent):
    """A sequence's first tokens have scores of -1e12, the later ones of size one."""
    print(f"[tree] range rising {fmt} {tile} 2^{exponent}", flush=True)
    c = case(hq, fmt, tile, [400, 90, 1500], [9, 20, 30], seed=46, pool=120)
    blocks = [-(-n // 32) for n in c.lens[:3]]
    for b, n in enumerate(blocks):  # blocks of their own
        c.table[b, :n] = torch.arange(n) + sum(blocks[:b])
    assert sum(blocks) <= 120
    g = torch.Generator().manual_seed(5)
    scale = torch.full((120, 32), 0.2)
    for b, n in enumerate(blocks):
        scale[sum(blocks[:b]):sum(blocks[:b]) + n // 2] = 1e12
    code = {"int8": -1, "e4m3": 0xB8, "mxfp4": 0xAA}[fmt]  # -1
    c.kc.codes.copy_(torch.full(c.kc.codes.shape, code, dtype=torch.int32).to(c.kc.codes.dtype))
    if fmt == "mxfp4":
        c.kc.scales.copy_(torch.where(scale > 1, 167, 125).to(torch.uint8)[:, None, :, None].expand(c.kc.scales.shape))
    else:
        c.kc.scales.copy_((scale * (0.5 + torch.rand(scale.shape, generator=g)))[:, None].expand(c.kc.scales.shape))
    d = torch.from_numpy(R.signs(R.SEED_K, 2 * N)).float().view(2, 1, N).expand(2, 4, N).reshape(1, 8, N)
    c.q, c.scale = d.expand(c.q.shape).contiguous(), 1.0
    set_scales(c.vc, exponent + torch.randint(-3, 4, (120, 32), generator=g))
    out = c.run().cpu().numpy()
    ref, _ = c.reference()
    for b in range(3):
        r = slice(c.starts[b], c.starts[b + 1])
        # scores of the tokens that count are below one: 2 * 150 U of it in a weight
        big = np.abs(R.values(c.vc)[c.table[b, :blocks[b]].numpy()]).max()
        assert (np.abs(out[r] - ref[r]) <= (c.lens[b] + 60 + 300) * U * big).all() and np.abs(ref[r]).max() > 1e-3 * big


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("low", [96, 0])
@pytest.mark.parametrize("side", ["k", "v", "both"])
def test_mxfp4_blocks_far_apart(hq, tile, low, side):
    """Block scales of a vector from 2^(low - 127) to 2^2: a code enters as a multiple of 2^-24 of the vector's
    largest block scale, half a step of which, 2^-25 of it, is a fourth of the U of the largest value
    that the bound allows for each token."""
    print(f"[tree] range blocks {tile} {low} {side}", flush=True)
    c = case(hq, "mxfp4", tile, [400, 90, 1500], [9, 20, 30], seed=47)
    g = torch.Generator().manual_seed(low)
    for x, of in ((c.kc, "k"), (c.vc, "v")):
        if side in (of, "both"):
            x.scales.copy_(torch.randint(low, 130, x.scales.shape, generator=g, dtype=torch.uint8))
            x.scales[::3, :, ::2, 1:] = 0  # one block alone counts
    c.vc.scales[:, :, ::7] = 0 if side != "k" else c.vc.scales[:, :, ::7]  # vectors of the least scale
    out = c.run()
    W.check(out.cpu().numpy(), *c.reference())
    assert torch.equal(c.run(), out) and c.kc.read_stats()["status"] == 0


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("below", [10, 14, 16, 20, 23, 25, 30])
def test_mxfp4_codes_of_a_block_far_below(hq, tile, below):
    """A sequence of one token, whose weight is 1: what comes out are its codes, in a block 2^-below of the
    largest one (which holds zeros) rounded to multiples of 2^-24."""
    c = case(hq, "mxfp4", tile, [1], [1], seed=48)
    blk = int(c.table[0, 0])
    g = torch.Generator().manual_seed(below)
    codes = torch.randint(0, 256, (2, 64), generator=g, dtype=torch.uint8)
    codes[:, :16] = 0
    c.vc.codes[blk, :, 0] = codes.cuda()
    c.vc.scales[blk, :, 0] = torch.tensor([127, 127 - below, 127 - below, 0], dtype=torch.uint8).cuda()
    out = c.run()[0].cpu().numpy().astype(np.float64).reshape(2, 4, N)
    y = (out * R.signs(R.SEED_V, 2 * N).reshape(2, 1, N)) @ R.hadamard()
    want = R.values(c.vc)[blk, :, 0]
    # half a step, and a handful of roundings of what came through the transform, sqrt(128) of its norm at most
    room = 2.0 ** -25 + 16 * U * np.linalg.norm(want, axis=-1).max() * np.sqrt(N)
    assert (np.abs(y - want[:, None]) <= room).all()
    assert below > 24 or np.abs(y).max() > 2.0 ** -below
