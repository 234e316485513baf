"""Rotary positions and attention with any visibility over the fixed-rate cache in plain
64-bit numpy, from their definitions in include/hq.h, with the bounds on how far fp32 kernels
may be off (beside tests/cache64.py)."""
import numpy as np
import torch

from tests.cache64 import N, SEED_K, SEED_V, U, hadamard, signs


def turn(x, table, positions, axis, interleaved, transposed=False):
    """x [rows, heads, 128] turned, and the bound on its fp32 error: two products and their sum,
    rounded once each.  Rows whose positions are not all in the table stay as they are."""
    x = x.astype(np.float64)
    y, tol = x.copy(), np.zeros_like(x)
    d, pairs = 2 * table.shape[2], table.shape[2]
    ok = ((positions >= 0) & (positions < table.shape[0])).all(1)
    for r in np.nonzero(ok)[0]:
        p = positions[r, axis]
        c, s = (table[p, i, np.arange(pairs)].astype(np.float64) for i in (0, 1))
        s = -s if transposed else s
        ia, ib = (np.arange(0, d, 2), np.arange(1, d, 2)) if interleaved else (np.arange(pairs), np.arange(pairs, d))
        a, b = x[r][:, ia], x[r][:, ib]
        y[r][:, ia], y[r][:, ib] = a * c - b * s, b * c + a * s
        tol[r][:, ia] = 2 * U * (np.abs(a * c) + np.abs(b * s)) + 1e-44
        tol[r][:, ib] = 2 * U * (np.abs(b * c) + np.abs(a * s)) + 1e-44
    return y, tol, ok


def visible(n, window, sinks):
    """The tokens that the newest of n sees."""
    t = np.arange(n)
    return (t >= n - window) | (t < sinks)


def tree_visible(n, masks, window=0, sinks=0):
    """[rows, n]: what the last len(masks) tokens of a sequence of n see."""
    rows = len(masks)
    ctx = n - rows
    live = np.zeros((rows, n), dtype=bool)
    for i, m in enumerate(masks):
        m = int(m) & ((1 << rows) - 1)
        t = np.arange(ctx)
        live[i, :ctx] = True if not window else (t >= ctx + bin(m).count("1") - window) | (t < sinks)
        live[i, ctx:] = [m >> j & 1 for j in range(rows)]
    return live


def attend(q, kv, vv, blocks, live, bt, scale, heads, group):
    """Rows q [rows, heads_q, 128] of one sequence whose tokens lie in `blocks` over the tokens
    that each sees, live [rows, n], in 64 bits, and the largest error that the kernels may make:
    as cache64.attend, with 8 U more for a query and 8 U more for a weight (22 of fp32's 24 bits
    enter a product; one-token attention has all of them)."""
    rows, n = live.shape
    H = hadamard()
    dk, dv = signs(SEED_K, heads * N).reshape(heads, N), signs(SEED_V, heads * N).reshape(heads, N)
    t = np.nonzero(live.any(0))[0]
    blk = blocks[t // bt]
    ok = (blk >= 0) & (blk < kv.shape[0])
    t, blk = t[ok], blk[ok]
    out, tol = np.zeros((rows, heads, group, N)), np.full((rows, heads, group, 1), 1e-30)
    qh = q.astype(np.float64).reshape(rows, heads, group, N)
    if not len(t):
        return out.reshape(rows, heads * group, N), np.broadcast_to(tol, out.shape).reshape(rows, heads * group, N)
    seen = live[:, t]
    for h in range(heads):
        k, v = kv[blk, h, t % bt], vv[blk, h, t % bt]
        qt = ((qh[:, h] * dk[h]) @ H).reshape(rows * group, N)
        s = (scale / N * (qt @ k.T)).reshape(rows, group, -1)
        big = np.sqrt((v * v).sum(-1) / N)
        mag = (np.abs(scale) / N * (np.abs(qt) @ np.abs(k).T)).reshape(s.shape)
        for i in range(rows):
            at = seen[i]
            if not at.any():
                continue
            p = np.exp(s[i][:, at] - s[i][:, at].max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[i, h] = ((p @ v[at]) @ H) / N * dv[h]
            m = mag[i][:, at].max(-1, keepdims=True) + np.abs(s[i][:, at]).max(-1, keepdims=True)
            tol[i, h] = (2 * 150 * U * m + (at.sum() + 60) * U) * big[at].max() + 1e-30
    return out.reshape(rows, heads * group, N), np.broadcast_to(tol, out.shape).reshape(rows, heads * group, N)


def check(got, ref, tol, scale=N ** -0.5):
    """Every value within its bound, and all together within what independent roundings leave."""
    off = np.abs(got - ref)
    assert (off <= tol).all(), float((off / np.maximum(tol, 1e-300)).max())  # a NaN is not
    size = np.linalg.norm(ref)
    assert np.linalg.norm(off) <= 64 * U * max(1.0, abs(scale) * N ** 0.5) * size + 1e-30


def random_tree(rng, n):
    """Ancestor masks (with themselves) of n tokens whose parents are drawn among those before."""
    masks = []
    for i in range(n):
        parent = int(rng.integers(-1, i))
        masks.append((1 << i) | (masks[parent] if parent >= 0 else 0))
    return masks


def mask_tensor(masks):
    return torch.from_numpy(np.array([int(m) for m in masks], dtype=np.uint64).view(np.int64))
