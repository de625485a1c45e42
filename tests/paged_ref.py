"""The operators of the paged cache and of drafts from their definitions, in 64 bits on the CPU, one row and one head at a time: nothing here is shared with
the library."""
import math

import numpy as np


def rope_angles(max_pos, rot, theta=1e4):
    """[max_pos][rot / 2] float64"""
    return np.arange(max_pos)[:, None] * theta ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))


def rotate(x, angle, pairs):
    """x [..., d] float64, angle [rot / 2]"""
    rot, out = 2 * len(angle), x.copy()
    one, two = (np.arange(rot // 2), np.arange(rot // 2) + rot // 2) if pairs == "halves" else (np.arange(0, rot, 2), np.arange(1, rot, 2))
    c, s = np.cos(angle), np.sin(angle)
    out[..., one], out[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    return out


def normed(x, w, eps):
    return x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * w


def place(table, n_pages, page, seq, slot):
    """(page, slot in it), or None for a hole"""
    p = int(table[seq, slot // page])
    return (p, slot % page) if 0 <= p < n_pages else None


def attention(q, k, v, seen):
    """q [nq][d], k and v [nkv][slots][d], seen: slots, float64.  Returns (out [nq][d], sum p |v|, sum |v| over the slots seen)."""
    nq, d = q.shape
    out, size, total = (np.zeros((nq, d)) for _ in range(3))
    for h in range(nq if len(seen) else 0):
        kv = h // (nq // k.shape[0])
        s = k[kv, seen] @ q[h] / math.sqrt(d)
        p = np.exp(s - s.max())
        p /= p.sum()
        out[h], size[h], total[h] = p @ v[kv, seen], p @ np.abs(v[kv, seen]), np.abs(v[kv, seen]).sum(0)
    return out, size, total


def branch(parents, i):
    got = []
    while True:
        got.append(i)
        if i == 0:
            return got[::-1]
        i = parents[i]


def softmax(x, T):
    e = np.exp((x - x.max()) / T)
    return e / e.sum()


def proper(x, T):
    return not np.isnan(x).any() and x.max() > -np.inf and (T == 0 or x.max() < np.inf)


def verify(parents, tokens, target, draft, T, accept, sample, width=64):
    """The verdict over one sequence: (rows that stay, next token).  Logits float64 [rows][vocab], draft may be None."""
    node, path, vocab = 0, [], target.shape[1]
    while True:
        after = [i for i in range(node + 1, len(parents)) if parents[i] == node][:width]
        with_q = draft is not None and T > 0 and after
        if not proper(target[node], T) or (with_q and not proper(draft[node], T)):
            return path, -1
        if T == 0:
            best = int(np.argmax(target[node]))
            onto = next((i for i in after if tokens[i] == best), None)
            if onto is None:
                return path, best
        else:
            p = whole = softmax(target[node], T)
            q = softmax(draft[node], T) if with_q else None
            onto = None
            for i in after:
                t = int(tokens[i])
                if not 0 <= t < vocab:
                    if q is not None:                 # what follows is drawn from what is left as after any failure
                        p = left_over(p, q)
                    continue
                if accept[i] * (q[t] if q is not None else 1.0) < p[t]:
                    onto = i
                    break
                if q is not None:
                    p = left_over(p, q)
                else:
                    p = p.copy()
                    p[t] = 0.0
                    p = p / p.sum() if p.sum() > 0 else p
            if onto is None:
                if not p.sum() > 0:
                    p = whole
                sums = np.cumsum(p)
                passes = np.nonzero((sums > sample * sums[-1]) & (p > 0))[0]
                return path, int(passes[0]) if len(passes) else int(np.nonzero(p)[0][-1])
        path.append(onto)
        node = onto


def left_over(p, q):
    p = np.maximum(p - q, 0.0)
    return p / p.sum() if p.sum() > 0 else p
