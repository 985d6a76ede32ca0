"""float64 oracle of the drafted-token operators: a tree's ancestors, rotary positions, rows in 8 bits,
attention over cached rows and ancestors, verification at given random numbers, and the accepted path's
move. Written from the definitions in the C header, one node or one row at a time."""
from __future__ import annotations

import math

import numpy as np

QMAX = {"int8": 127.0, "e4m3": 448.0}


def lines(parent, T, room=None):
    """Per node its ancestors and itself in order, or None for an absent node. room: nodes that fit the cache."""
    out = []
    for t in range(T):
        p = t - 1 if parent is None else int(parent[t])
        if room is not None and t >= room:
            out.append(None)
        elif p == -1:
            out.append([t])
        elif 0 <= p < t and out[p] is not None:
            out.append(out[p] + [t])
        else:
            out.append(None)
    return out


def frequencies(rot, theta, scaling="none", factor=1.0, low=1.0, high=4.0, orig_len=8192):
    f = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "wavelength":
        out = []
        for x in f:
            g = min(1.0, max(0.0, (orig_len * x / (2 * math.pi) - low) / (high - low)))
            out.append(x * (g + (1 - g) / factor))
        return out
    if scaling == "index":
        at = lambda turns: rot * math.log(orig_len / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
        a, b = max(0, math.floor(at(high))), min(rot - 1, math.ceil(at(low)))
        out = []
        for i, x in enumerate(f):
            g = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            out.append(x * ((1 - g) + g / factor))
        return out
    return f


def rotate(x, pos, layout, rot, freq, mscale=1.0):
    """One head vector (float64) turned by position pos."""
    y = np.array(x, np.float64)
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = math.cos(pos * freq[i]) * mscale, math.sin(pos * freq[i]) * mscale
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def attention(q, k, v, seen, scale):
    """One query over the rows `seen` of k, v (float64): (output, sum of p |v|)."""
    if len(seen) == 0:
        return np.zeros(v.shape[1]), np.zeros(v.shape[1])
    s = k[seen] @ q * scale
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ v[seen], p @ np.abs(v[seen])


def softmax(l, temperature):
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    m = l.max()
    if m == -np.inf:
        return None
    with np.errstate(invalid="ignore"):
        e = np.where(l == m, 1.0, np.exp((l - m) / temperature))
    return e / e.sum()


def verify(logits, tokens, u, parent=None, draft=None, temperature=1.0):
    """One tree: (ids, path) without padding. Probabilities are updated child by child, as the definition has it."""
    T, V = logits.shape
    line = lines(parent, T)
    up = [None if line[t] is None else -1 if len(line[t]) == 1 else line[t][-2] for t in range(T)]
    dist = []
    for t in range(T):
        if temperature == 0:
            l = np.where(np.isnan(logits[t]), -np.inf, logits[t])
            dist.append(np.eye(1, V, int(np.argmax(l)))[0] if l.max() > -np.inf else None)
        else:
            dist.append(softmax(logits[t], temperature))
    node, path, ids = 0, [0], []
    while True:
        p = dist[node]
        kids = [t for t in range(1, T) if up[t] == node]
        if p is None:
            return ids + [-1], path
        full, taken = p, None
        for c in kids:
            x = int(tokens[c])
            if draft is not None and temperature > 0:
                q = softmax(draft[node], temperature)
                if 0 <= x < V and (0.0 if q is None else u[c] * q[x]) < p[x]:
                    taken = c
                    break
                p = np.maximum(p - (0.0 if q is None else q), 0.0)
            else:
                left = p.sum()
                if 0 <= x < V and u[c] * left < p[x] if temperature else 0 <= x < V and p[x] > 0:
                    taken = c
                    break
                if 0 <= x < V:
                    p = p.copy()
                    p[x] = 0.0
        if taken is None:
            break
        ids.append(int(tokens[taken]))
        path.append(taken)
        node = taken
    if temperature == 0:
        return ids + [int(np.argmax(full))], path
    if p.sum() <= 0:
        p = full
    cum = np.cumsum(p)
    hit = np.nonzero(cum > u[0] * cum[-1])[0]
    return ids + [int(hit[0]) if len(hit) else int(np.nonzero(p)[0][-1])], path
