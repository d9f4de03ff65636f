"""Pins of the oracle of growing nodes, projections and token log probabilities (oracle/step.py), and what the entry points
refuse without a handle."""
import math

import numpy as np
import pytest
import torch

from oracle import step as OS


def test_slots_worked_by_hand():
    o = OS.OpenNodes()
    o.open(4, 70, 128)
    o.open(2, 3, 0)
    assert o.append([4, 2], None, [2, 3], 5) == ([128, 129, 0, 1, 2], [2, 3])
    assert o.append([2, 4], None, [1, 1], 2) == ([-1, 130], [-1, 3])          # node 2 has no room
    assert o.append([4], [1], [2], 4) == ([129, 130, -1, -1], [3])            # one token stays, two are replaced; rows behind the last
    assert o.append([9, 4], None, [1, -1], 2) == ([-1, -1], [-1, -1])         # not open; a negative count takes no rows
    assert o.append([4, 2], [4, 1], [0, 0], 0) == ([], [-1, 1])               # holds only three; taken back to one
    assert o.append([2, 4], None, [1, 2], 2) == ([1, -1], [2, -1])            # rows beyond num_new


def test_projection_by_matrices():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((3, 5)), rng.standard_normal((4, 5))
    a, b, f = rng.standard_normal((2, 2, 5)), rng.standard_normal((2, 4, 2)), np.array([0.5, -2.0])
    y, size = OS.project(x, w, a, b, f, [1, -1, 0])
    assert np.allclose(y[0], (w - 2 * b[1] @ a[1]) @ x[0]) and np.allclose(y[1], w @ x[1]) and np.allclose(y[2], (w + 0.5 * b[0] @ a[0]) @ x[2])
    assert np.all(size >= np.abs(y))


def test_logprobs_against_torch_and_closed_forms():
    rng = np.random.default_rng(2)
    x = rng.standard_normal(50)
    lp, h, lse, ids, tops = OS.token_logprobs(x.tolist(), 7, 5)
    t = torch.distributions.Categorical(logits=torch.from_numpy(x))
    assert math.isclose(lp, float(t.logits[7])) and math.isclose(h, float(t.entropy())) and math.isclose(lse, float(torch.logsumexp(torch.from_numpy(x), 0)))
    assert ids == torch.topk(torch.from_numpy(x), 5).indices.tolist() and np.allclose(tops, t.logits[ids].numpy())
    assert OS.token_logprobs([1.0] * 8, 3, 3)[:2] == pytest.approx((-math.log(8), math.log(8))) and OS.token_logprobs([1.0] * 8, 3, 3)[3] == [0, 1, 2]
    assert OS.token_logprobs([-math.inf, 2.0], 1, 2) == (0.0, 0.0, 2.0, [1, 0], [0.0, -math.inf])
    assert OS.token_logprobs([-math.inf] * 3, 1, 1) == (-math.inf, 0.0, -math.inf, [0], [-math.inf])
    assert OS.token_logprobs([0.0, -0.0, math.nan, -math.inf], -1, 4)[3] == [0, 1, 3, 2] and math.isnan(OS.token_logprobs([math.inf, 0.0], 0, 1)[1])


def test_refusals_without_a_handle():
    from paper_2605_22566_b200 import binding as B
    p = B.ProjectionDesc(64, 8, 1 << 20, 64, 0, 0, None, None, None)
    assert B.gf_node_kv_open(None, 0, 1) == B.gf_node_kv_close(None, 0, 1) == B.GF_ERR_INVALID_ARG
    assert B.gf_append_slots(None, 1, 16, None, 16, 1, 16) == B.gf_node_kv_append(None, 0, 1, 16, 16, 64, 16, 64) == B.GF_ERR_INVALID_ARG
    assert B.gf_adapter_project(None, p, 1, 16, 64, None, 16, 8, 0) == B.GF_ERR_INVALID_ARG
    assert B.gf_token_logprobs(None, 1, 8, 16, 8, 0, None, 0, B.Logprobs()) == B.GF_ERR_INVALID_ARG
    assert B.gf_adapter_project_scratch_bytes(p, 4) == 0                                                   # no adapters
    p = B.ProjectionDesc(1032, 8, 1 << 20, 1032, 2, 24, 1 << 20, 1 << 20, None)
    assert B.gf_adapter_project_scratch_bytes(p, 4) >= 4 * 24 * 4 and B.gf_adapter_project_scratch_bytes(p, 0) == 0
    for bad in (dict(in_dim=1030), dict(out_dim=0), dict(w_stride=1024), dict(w_stride=1036), dict(rank=72), dict(rank=12), dict(w_dev=(1 << 20) + 8),
                dict(a_dev=None), dict(b_dev=(1 << 20) + 2), dict(num_adapters=-1), dict(scale_dev=2)):
        q = B.ProjectionDesc(*[bad.get(n, getattr(p, n)) for n, _ in p._fields_])
        assert B.gf_adapter_project_scratch_bytes(q, 4) == 0, bad


def test_sizes_next_to_the_end_of_int32_are_refused():
    from paper_2605_22566_b200 import binding as B
    p = B.ProjectionDesc(1032, 8, 1 << 20, 1032, 2, 24, 1 << 20, 1 << 20, None)
    assert B.gf_adapter_project_scratch_bytes(p, 2 ** 31 - 512) > 0
    assert B.gf_adapter_project_scratch_bytes(p, 2 ** 31 - 511) == B.gf_adapter_project_scratch_bytes(p, 2 ** 31 - 1) == 0
    for out_dim, ok in ((2 ** 31 - 512, True), (2 ** 31 - 511, False), (2 ** 31 - 1, False)):
        q = B.ProjectionDesc(*[out_dim if n == "out_dim" else getattr(p, n) for n, _ in p._fields_])
        assert (B.gf_adapter_project_scratch_bytes(q, 4) > 0) == ok
    q = B.ProjectionDesc(*[{"in_dim": 2 ** 30 + 8, "w_stride": 2 ** 30 + 8}.get(n, getattr(p, n)) for n, _ in p._fields_])
    assert B.gf_adapter_project_scratch_bytes(q, 4) == 0
