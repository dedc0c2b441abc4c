"""Attention of a tree of drafted tokens over a KV cache, and the norm and
rotation in front of it, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

What is computed
----------------
A draft proposes n nodes behind a sequence of L tokens; node i's parent is an
earlier node or -1 (the sequence's last token).  A node of depth d (its number
of ancestors) lies at index L + d of its own path.  It attends to the
sequence's tokens 0 .. L - 1, to its ancestors and to itself; with a window of
W keys only to those of them whose index on the node's path is above L + d - W,
or below ``first``.  Each node's output is the attention of
``attention.attention`` over exactly those keys.

``norm_rotate``: y = x w / sqrt(mean x^2 + eps) per head, then the first
``rot`` channels turn in pairs (i, i + rot / 2), or (2 i, 2 i + 1), by the
angle position * inv_freq[i]:  (a, b) -> (a cos - b sin, b cos + a sin) mscale.
"""

from __future__ import annotations

import numpy as np

from . import attention as _att


def depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def path_to(parents, i):
    """Node i's ancestors and itself, from the root on."""
    path = []
    while i >= 0:
        path.append(i)
        i = parents[i]
    return path[::-1]


def visible(parents, length, window=0, first=0, keep=None):
    """Per node, the slots (cache indices, then length + node) it attends to."""
    out = []
    for i in range(len(parents)):
        path = path_to(parents, i)
        here = length + len(path) - 1
        slots = [(t, t) for t in range(length) if keep is None or keep[t]]
        slots += [(length + d, length + node) for d, node in enumerate(path)]
        out.append([slot for index, slot in slots
                    if not window or index > here - window or index < first])
    return out


def draft_attention(q, k, v, parents, scale, group, window=0, first=0, sinks=None, keep=None):
    """q [n, Hq, D]; k, v [L + n, Hkv, D] (the cache, then the nodes): [n, Hq, D]."""
    length = k.shape[0] - len(parents)
    seen = visible(parents, length, window, first, keep)
    return np.stack([_att.attention(np.asarray(q[i], dtype=np.float64), k[s], v[s], scale, group, None, sinks)
                     for i, s in enumerate(seen)])


def norm_rotate(x, positions, inv_freq=None, weight=None, eps=0.0, interleaved=False, mscale=1.0):
    """x [n, heads, D] -> [n, heads, D], all in float64."""
    y = np.asarray(x, dtype=np.float64).copy()
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + float(eps)) * np.asarray(weight, dtype=np.float64)
    if inv_freq is None:
        return y
    f = np.asarray(inv_freq, dtype=np.float64)
    rot = 2 * len(f)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * f
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    i = np.arange(len(f))
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    z = y.copy()
    z[..., a] = (y[..., a] * cos - y[..., b] * sin) * mscale
    z[..., b] = (y[..., b] * cos + y[..., a] * sin) * mscale
    return z
