"""The gate's gradient behind a norm with a bias, where what it multiplies nearly vanishes in a channel."""
import numpy as np
import pytest
import torch

from between_util import DEPTH, kept
from layer_grads_util import U32, f64, half_step, least
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
SEED = 11


@pytest.mark.parametrize("n, width, p", [(7, 40, 0.0), (900, 200, 0.1), (5000, 1000, 0.1), (3000, 2050, 0.0)])
@pytest.mark.parametrize("weight", [1.0, -30.0])
def test_channels_that_nearly_cancel(n, width, p, weight):
    """Every fifth channel has the same large value in all rows, so that its normed value hardly moves, and a bias that takes it away.  The
    gradient is weight * sum_t D N(x) + bias * sum_t D: off by what fp32 leaves in the two sums, and no more."""
    g = torch.Generator().manual_seed(n)
    x, dh = torch.randn(n, width, generator=g), torch.randn(n, width, generator=g).abs()
    x[:, ::5] = 50.0
    t = f64(x)
    hat = t / np.sqrt((t * t).mean(1, keepdims=True) + 1e-5)
    params = torch.cat([torch.full((width,), weight), torch.from_numpy(-weight * hat.mean(0)).float(), torch.ones(width)])
    params[width:2 * width][1::5] = 0.25
    form = B.Join(width, torch.float32, norm="rms", after=True, before=False, after_weight=0, after_bias=width, gate=2 * width, dropout=p, seed=SEED)
    grad = torch.zeros(3 * width, device="cuda")
    B.adasum_join_grad(form, params.cuda(), grad, x=x.cuda(), dh=dh.cuda(), dresidual=False)
    d = f64(dh)
    if p:
        mask, factor = kept(n, width, p, SEED)
        d = np.where(mask, d * factor, 0.0)
    w, b = f64(params[:width]), f64(params[width:2 * width])
    want = (d * (hat * w + b)).sum(0)
    # D and N(x) carry a few roundings and those of a row's statistics; a lane adds up to n / 256 rows in fp32, its workgroup's sum is rounded
    # to fp32, the rest is fp64
    off = (DEPTH + -(-n // 256) + 2 + 8) * U32
    tol = off * (np.abs(w) * np.abs(d * hat).sum(0) + np.abs(b) * np.abs(d).sum(0)) + half_step(torch.float32) * np.abs(want) + least(torch.float32)
    assert (np.abs(f64(grad[2 * width:]) - want) <= tol).all()
    # (the sums are a hundred times what is left of them where it matters)
    assert (np.abs(w * (d * hat).sum(0)) > 30 * np.abs(want))[::5].mean() > 0.9
