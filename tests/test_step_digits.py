"""That the bounds of step_digits.py tell the arithmetic that is meant from the next coarser one (planted here, on the host)."""
import numpy as np
import pytest
import torch

import step_digits as D


@pytest.mark.parametrize("k", [512, 1024, 2048, 16384])
def test_sums_that_are_not_taken_out_are_seen(k):
    x, w = D.same_sign(6, k, 40)
    exact = x.double().numpy() @ w.double().numpy().T
    off = lambda y: np.linalg.norm(y - exact) / np.linalg.norm(exact)  # noqa: E731
    assert off(D.sums_cut_off(x, w, D.CHUNK_K)) < 0.8 * D.SAME_SIGN
    if k >= 2048:
        assert off(D.sums_cut_off(x, w, k)) > 1.5 * D.SAME_SIGN


def test_a_number_less_is_seen():
    x, a, b = D.between_numbers(40, 30, 2, 16)
    h = (x.double() @ a[0].double().T)
    assert torch.equal(h, h.float().double())
    exact = h @ b[0].double().T
    off = [float(((D.in_numbers(h, m) @ b[0].double().T - exact).abs() / exact).max()) for m in (1, 2, 3)]
    assert off[2] == 0.0 and 1.5 * D.THREE < off[1] < D.TWO and off[0] > 100 * D.TWO


def test_what_is_left_of_two_parts_that_cancel():
    x, a, b = D.between_numbers(40, 30, 1, 24)
    w = D.cancelling(x, b[0])
    assert w.shape == (30, x.shape[1]) and not w.isnan().any()
    adapter = (x.double() @ a[0].double().T) @ b[0].double().T
    y = x.double() @ w.double().T + adapter
    assert float((y / adapter).min()) > 2.0 ** -19 and float((y / adapter).max()) < 2.0 ** -17
