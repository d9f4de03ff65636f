"""fp64 definition of accumulated attention weights and of the tokens that an eviction keeps.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


def attention_weights(paths, node_kv, q, lse, num_kv_heads, scale=None):
    """{node: [Hkv, tokens]}: per token the sum over the requests whose path holds its node, and the query
    heads of the KV head, of exp(scale <q, k> - lse)."""
    R, Hq, D = q.shape
    g = Hq // num_kv_heads
    sc = 1.0 / np.sqrt(D) if scale is None else scale
    out = {}
    for r in range(R):
        for v in paths[r]:
            K = node_kv(v)[0]
            w = out.setdefault(v, np.zeros((num_kv_heads, K.shape[0])))
            for h in range(Hq):
                w[h // g] += np.exp(K[:, h // g, :] @ q[r, h] * sc - lse[r, h])
    return out


def kept(weights, keep, first, last):
    """Ascending indices of the tokens kept of one (layer, KV head): by a sort of explicit keys."""
    n = len(weights)
    m = min(n, keep)

    def key(t):
        w = float(weights[t])
        if t < first or t >= n - last:
            return (0, 0.0, t)
        return (1, math.inf if math.isnan(w) else -w, t) if not math.isnan(w) else (2, 0.0, t)
    return sorted(sorted(range(n), key=key)[:m])
