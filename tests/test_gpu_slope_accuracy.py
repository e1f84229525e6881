"""gelu's slope far from zero: how near it comes to the definition, relative to its own terms."""
import numpy as np
import pytest
import torch

from layer_grads_util import f64, phi
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


def slopes(x):
    """The kept values of a column (a block of its own each) and gelu's slopes there."""
    kept = B.adasum_checkpoint_store(x[:, None].cuda())
    got = B.adasum_checkpoint_act_grad(kept, torch.ones(x.numel(), 1, device="cuda"), "gelu")
    return f64(B.adasum_checkpoint_load(kept))[:, 0], f64(got)[:, 0]


@pytest.mark.parametrize("lo, hi", [(1e-3, 2), (2, 4), (4, 6), (6, 9), (9, 12.5)])
def test_gelu_slope_relative_to_its_terms(lo, hi):
    v, got = slopes(-torch.linspace(lo, hi, 4001))
    tail, density = phi(v)
    # f(a) (M(a) - a): the exponential and its correction take 2 and 1 half steps, M 6 (a reciprocal of 2, its argument and the polynomial's
    # last steps), the difference and the product 1 each, the constants 1: 12, at most, of the sum of the two terms
    assert (np.abs(got - (tail + v * density)) <= 16 * 2.0 ** -24 * (tail - v * density)).all()
    # at the positive value it is one minus that
    w, got = slopes(torch.linspace(lo, hi, 4001))
    assert np.array_equal(w, -v)
    assert (np.abs(got - (1 - (tail + v * density))) <= 2.0 ** -24 + 16 * 2.0 ** -24 * (tail - v * density)).all()


def test_gelu_slope_beyond_all_terms():
    v, got = slopes(torch.tensor([13.0, -13.0, 20.0, -20.0, 1e4, -1e4, 1e19, -1e19, 3e38, -3e38, float("inf"), float("nan"), 0.0, 1e-38]))
    want = [1, 0] * 5 + [float("nan")] * 2 + [0.5] * 2
    assert np.allclose(got, want, rtol=0, atol=1e-34, equal_nan=True)
