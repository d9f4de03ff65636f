"""fp64 / exact-integer definitions of what stands around a step's attention: growing nodes, projections with per-row
low-rank adapters, and what a row of logits says of its tokens.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


class OpenNodes:
    """Open nodes, one list of rows each: append puts rows behind the ones that stay."""

    def __init__(self):
        self.room, self.off, self.rows = {}, {}, {}

    def open(self, node, room, off):
        self.room[node], self.off[node], self.rows[node] = room, off, []

    def append(self, nodes, held, counts, num_new, rows=None):
        """held None: all.  (slots, lengths): -1 where a request is refused.  rows: what arrives, [num_new, ...]."""
        slots, lens, at, seen = [-1] * num_new, [], 0, set()
        for r, (v, c) in enumerate(zip(nodes, counts)):
            h = len(self.rows[v]) if held is None and v in self.rows else (0 if held is None else held[r])
            begin = at
            at += max(c, 0)
            again = v in seen  # (of requests that name the same node the first one counts)
            seen.add(v)
            if again or v not in self.rows or c < 0 or h < 0 or h > len(self.rows[v]) or at > num_new or h + c > self.room[v]:
                lens.append(-1)
                continue
            del self.rows[v][h:]
            for i in range(c):
                slots[begin + i] = self.off[v] + h + i
                self.rows[v].append(None if rows is None else rows[begin + i])
            lens.append(h + c)
        return slots, lens


def project(x, w, a=None, b=None, scale=None, adapters=None):
    """x [rows, in], w [out, in], a [n, rank, in], b [n, out, rank]: (y, what the sums of magnitudes are)."""
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if adapters is not None:
        for t, i in enumerate(adapters):
            if 0 <= i < len(a):
                f = 1.0 if scale is None else scale[i]
                y[t] += f * (b[i] @ (a[i] @ x[t]))
                size[t] += abs(f) * (np.abs(b[i]) @ (np.abs(a[i]) @ np.abs(x[t])))
    return y, size


def token_logprobs(row, token, top):
    """One row of logits: (logprob, entropy, lse, ids, their log probabilities)."""
    v = len(row)
    order = sorted(range(v), key=lambda i: (math.isnan(row[i]), 0.0 if math.isnan(row[i]) else -row[i], i))[:top]
    m = log_sum = 0.0
    if any(math.isnan(x) or x == math.inf for x in row):
        lse = entropy = math.nan
    elif max(row) == -math.inf:
        lse, entropy = -math.inf, 0.0
    else:
        m = max(row)
        log_sum = math.log(math.fsum(math.exp(x - m) for x in row))
        lse = m + log_sum
        # (relative to the largest, so that nothing is lost where all are large)
        entropy = math.fsum(math.exp(x - m - log_sum) * (log_sum - (x - m)) for x in row if math.exp(x - m - log_sum) > 0)

    def of(i):
        return lse if not math.isfinite(lse) else row[i] - m - log_sum
    logprob = 0.0 if token == -1 else of(token) if 0 <= token < v else math.nan
    return logprob, entropy, lse, order, [of(i) for i in order]
