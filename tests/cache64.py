"""The fixed-rate cache and the fused norm in plain 64-bit numpy, from their
definitions in include/hq.h, with the bounds on how far fp32 kernels may be off."""
import numpy as np
import torch

N = 128
U = 2.0 ** -24  # half a step of fp32, relative
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
TOP = {"int8": 127.0, "e4m3": 448.0}
SEED_K, SEED_V = 41, 51


def signs(seed, cols):
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + (np.arange(cols, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return np.where(z >> np.uint64(63), -1.0, 1.0)


def hadamard(n=N):
    h = np.ones((1, 1))
    while h.shape[0] < n:
        h = np.block([[h, h], [h, -h]])
    return h


def transform(x, seed, heads):
    """[..., heads * 128] -> y = H D x, [..., heads, 128], and the bound on an
    fp32 butterfly transform's error (seven stages of sums of |x|)."""
    xd = (x.astype(np.float64) * signs(seed, heads * N)).reshape(x.shape[:-1] + (heads, N))
    return xd @ hadamard(), 7 * U * np.abs(xd).sum(-1, keepdims=True)


def e4m3_values(b):
    b = b.astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e > 0, 2.0 ** (e - 10) * (8 + m), 2.0 ** -9 * m)
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(b >= 128, -v, v)


def values(cache):
    """What every slot of a cache stands for in the stored coordinates:
    [blocks, heads, block_tokens, 128]."""
    codes, scales = cache.codes.cpu().numpy(), cache.scales.cpu().numpy()
    fmt = name(cache)
    if fmt == "mxfp4":
        nib = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (N,))
        v = np.where(nib >= 8, -1.0, 1.0) * E2M1[nib & 7]
        f = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return v * np.repeat(f, 32, -1)
    c = codes.astype(np.float64) if fmt == "int8" else e4m3_values(codes.view(np.uint8))
    return c * scales.astype(np.float64)[..., None]


def name(cache):
    return {3: "int8", 4: "e4m3", 5: "mxfp4"}[cache.format]


def rows_of(cache, seed, slots):
    """The rows that slots stand for, D H (s c) / 128, [rows, heads * 128]."""
    v = values(cache)[slots // cache.block_tokens, :, slots % cache.block_tokens]
    return (v @ hadamard() / N).reshape(len(slots), -1) * signs(seed, cache.heads * N)


def check_codes(fmt, y, err, got):
    """Stored values `got` are y cast to the format: within half a step of the
    cast plus what fp32 may move y by (the scale and the product round once each:
    4 U of the value, and of the scale's step)."""
    amax = np.abs(y).max(-1, keepdims=True)
    if fmt == "int8":
        half = amax / 127 / 2
    elif fmt == "e4m3":
        half = np.maximum(np.abs(y) * 2.0 ** -4, amax / 448 * 2.0 ** -10)
    else:
        b = y.reshape(y.shape[:-1] + (4, 32))
        x = np.floor(np.log2(np.abs(b).max(-1, keepdims=True).clip(1e-30))) - 2
        # an fp32 y may lie on the other side of a power of two: the step is then half or
        # twice as large; only blocks that near one get the larger step
        m = np.abs(b).max(-1, keepdims=True)
        near = m * (1 + 1e-5) >= 2.0 ** (x + 3)
        t = np.abs(b) / 2.0 ** x
        step = np.where(t <= 2, .25, np.where(t <= 4, .5, np.where(t <= 6, 1.0, t - 6)))
        half = (np.where(near, 2 * np.maximum(step, .5), step) * 2.0 ** x).reshape(y.shape)
    off = np.abs(got - y)
    room = half * (1 + 8 * U) + 2 * err + 8 * U * amax
    assert (off <= room).all(), (fmt, float((off - room).max()), float(amax.max()))


def attend(q, kv, vv, table, lens, bt, scale, heads, group):
    """64-bit attention over caches given as values() and the largest error that
    fp32 may make: scores are sums of 128 products (a bound of 140 U of the sum of
    magnitudes: the query's transform, its scaling, the products), which the
    softmax turns into a relative error of twice that, and the value sums of T
    terms, their joins and the output's transform add (T + 40) U."""
    B = q.shape[0]
    H = hadamard()
    dk, dv = signs(SEED_K, heads * N).reshape(heads, N), signs(SEED_V, heads * N).reshape(heads, N)
    out, tol = np.zeros((B, heads, group, N)), np.zeros((B, heads, group, 1))
    qh = q.astype(np.float64).reshape(B, heads, group, N)
    for b in range(B):
        t = np.arange(lens[b])
        blk = table[b, t // bt]
        ok = (blk >= 0) & (blk < kv.shape[0])
        t, blk = t[ok], blk[ok]
        if not len(t):
            continue
        for h in range(heads):
            k, v = kv[blk, h, t % bt], vv[blk, h, t % bt]
            qt = (qh[b, h] * dk[h]) @ H
            s = scale / N * (qt @ k.T)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, h] = ((p @ v) @ H) / N * dv[h]
            mag = np.abs(scale) / N * (np.abs(qt) @ np.abs(k).T).max(-1, keepdims=True) + np.abs(s).max(-1, keepdims=True)
            # a coordinate of a row moved back is at most its norm / sqrt(128)
            big = np.sqrt((v * v).sum(-1).max() / N)
            tol[b, h] = (2 * 140 * U * mag + (len(t) + 40) * U) * big + 1e-30
    return out.reshape(B, heads * group, N), np.broadcast_to(tol, out.shape).reshape(B, heads * group, N)


def random_cache(hq, plan, fmt, blocks, heads, bt, seed, stale=False):
    """A cache with random contents in every slot."""
    g = torch.Generator().manual_seed(seed)
    c = hq.Cache(plan, blocks, bt, {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt], heads=heads)
    if fmt == "mxfp4":
        c.codes.copy_(torch.randint(0, 256, c.codes.shape, generator=g, dtype=torch.uint8))
        c.scales.copy_(torch.randint(126, 130, c.scales.shape, generator=g, dtype=torch.uint8))
        return c
    v = torch.randn(c.codes.shape, generator=g)
    c.scales.copy_(0.1 + 0.3 * torch.rand(c.scales.shape, generator=g))
    if fmt == "int8":
        c.codes.copy_((v * 40).round().clamp(-127, 127).to(torch.int8))
    else:
        c.codes.copy_((v * 30).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return c


def plans(hq, heads):
    cols = (heads * N + 511) // 512 * 512
    return hq.hq_plan(cols=cols, bps=4.0, rht_seed=SEED_K), hq.hq_plan(cols=cols, bps=4.0, rht_seed=SEED_V)
