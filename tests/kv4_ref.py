"""The 4-bit cache's operators from their definitions, in 64 bits on the CPU (numpy), one row and one head at a time: nothing here is shared with
the library."""
import math

import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def pack(codes):
    """[..., channels] of 4-bit codes -> bytes."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def quantise_group(x):
    """32 float64 values -> (codes, scale byte)."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(32, dtype=np.uint8), 255
    top = np.abs(x).max()
    s = -100
    if top > 0:
        s = math.ceil(math.log2(top / 7)) - 2
        while top > 7 * 2.0 ** s:
            s += 1
        s = min(max(s, -100), 125)
    a = np.abs(x) / 2.0 ** s
    code = np.zeros(32, dtype=np.uint8)
    for c in range(1, 8):
        middle = (LEVELS[c - 1] + LEVELS[c]) / 2
        code[(a > middle) | ((a == middle) & (c % 2 == 0))] = c
    return code | (np.signbit(x).astype(np.uint8) << 3), s + 127


def quantise(x):
    """float64 [..., d] -> (codes [..., d], scale bytes [..., d / 32])."""
    g = x.reshape(-1, 32)
    got = [quantise_group(r) for r in g]
    return (np.stack([c for c, _ in got]).reshape(x.shape),
            np.array([b for _, b in got], dtype=np.uint8).reshape(*x.shape[:-1], -1))


def values(codes, scales):
    """codes [..., d], scale bytes [..., d / 32] -> float64."""
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(*scales.shape, 32) * unit[..., None]).reshape(codes.shape)


def attention(q, k, v, length):
    """q [rows][nq][d], k and v [nkv][length + rows][d], float64.  Returns (out, sum of p |v|, weight of every slot [nkv][slots])."""
    rows, nq, d = q.shape
    nkv = k.shape[0]
    out, size = np.zeros((rows, nq, d)), np.zeros((rows, nq, d))
    got = np.zeros((nkv, k.shape[1]))
    for h in range(nq):
        kv = h // (nq // nkv)
        for i in range(rows):
            n = length + i + 1
            with np.errstate(invalid="ignore"):
                s = k[kv, :n] @ q[i, h] / math.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[i, h], size[i, h] = p @ v[kv, :n], p @ np.abs(v[kv, :n])
            got[kv, :n] += p
    return out, size, got


def evict(weights, positions, pos, keep, recent):
    """Slots that the first `keep` slots hold afterwards (one head; weights and positions of its slots)."""
    n = len(weights)
    if n <= keep:
        return list(range(n))
    def rank(i):
        if positions[i] >= pos - recent:
            return (0, 0.0, positions[i], i)
        w = float(weights[i])
        return (1, -w, positions[i], i) if not math.isnan(w) else (2, 0.0, positions[i], i)
    kept = set(sorted(range(n), key=rank)[:keep])
    late = iter(i for i in range(keep, n) if i in kept)
    return [i if i in kept else next(late) for i in range(keep)]
