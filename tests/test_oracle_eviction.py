"""Pins of the oracle of attention weights and eviction (oracle/eviction.py), and what the entry points refuse without a handle."""
import itertools

import numpy as np
import pytest

from oracle import attention as OA
from oracle import eviction as OE


def test_every_head_gives_away_one_and_a_nodes_share_is_split_among_its_tokens():
    rng = np.random.default_rng(1)
    kv = {v: (rng.standard_normal((n, 2, 8)), rng.standard_normal((n, 2, 8))) for v, n in ((0, 5), (1, 3), (2, 4))}
    paths = [[0, 1], [0, 2], [0]]
    q = rng.standard_normal((3, 4, 8))
    _, lse = OA.decode(paths, kv.__getitem__, q, 2)
    w = OE.attention_weights(paths, kv.__getitem__, q, lse, 2)
    assert np.isclose(sum(x.sum() for x in w.values()), 3 * 4)        # every (request, head) gives away 1
    # request 2 attends to node 0 alone, so that node gets at least its 4 heads' worth; equal keys get equal shares
    assert w[0].sum() >= 4.0
    kv[1] = (np.broadcast_to(kv[1][0][:1], kv[1][0].shape), kv[1][1])
    _, lse = OA.decode(paths, kv.__getitem__, q, 2)
    w = OE.attention_weights(paths, kv.__getitem__, q, lse, 2)
    assert np.allclose(w[1], w[1][:, :1])


def test_kept_by_brute_force_over_all_subsets():
    rng = np.random.default_rng(2)
    for _ in range(60):
        n = int(rng.integers(1, 8))
        w = rng.integers(0, 3, n).astype(float)
        first, last = int(rng.integers(0, 3)), int(rng.integers(0, 3))
        keep = first + last + int(rng.integers(0, 4))
        m = min(n, keep)
        must = {t for t in range(n) if t < first or t >= n - last}
        best = None
        for sub in itertools.combinations(range(n), m):  # lexicographic: among equal sums the earliest indices come first
            if len(must & set(sub)) < min(len(must), m):
                continue
            total = sum(w[t] for t in sub if t not in must)
            if best is None or total > best[0]:
                best = (total, list(sub))
        assert OE.kept(w, keep, first, last) == best[1]


def test_kept_orders_nan_last_and_infinities():
    w = np.array([np.nan, -np.inf, 0.0, np.inf, -0.0, 1.0])
    assert OE.kept(w, 2, 0, 0) == [3, 5]
    assert OE.kept(w, 3, 0, 0) == [2, 3, 5]          # +0 and -0 are equal: the lower index
    assert OE.kept(w, 5, 0, 0) == [1, 2, 3, 4, 5]
    assert OE.kept(w, 3, 1, 1) == [0, 3, 5]


@pytest.fixture(scope="module")
def B():
    from paper_2605_22566_b200 import build
    build.build()
    from paper_2605_22566_b200 import binding
    return binding


def test_refusals_without_a_handle(B):
    assert B.gf_kv4_bytes_per_tile(128) == 9216 and B.gf_kv4_bytes_per_tile(64) == 4608
    assert B.gf_kv4_pool_attach(None, 1 << 20, 1 << 20) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv4_write(None, 0, 0, 16, 16, 1) == B.GF_ERR_INVALID_ARG
    assert B.gf_weight_slots(None) == 0
    assert B.gf_path_attention_weights(None, None, 0, 16, 16, 1, 16) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_evict(None, [(0, 1, 2, 0, 0)], 16, 16) == B.GF_ERR_INVALID_ARG
    with pytest.raises(B.GfError):
        B.gf_kv4_pool_info(None)
