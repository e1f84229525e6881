"""Norms around a mean of rows of equal values, with an eps that any remainder of the mean would outweigh."""
import numpy as np
import pytest
import torch

from between_util import DEPTH
from layer_grads_util import U32, f64
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-12
VALUES = [3.0, 100.3, -0.1, 4097.0, 0.0, 1e-3, 7.0, 255.0]
WIDTHS = [1, 7, 33, 200, 300, 1000, 1023, 2047, 3000, 8191]


def rows(width):
    return torch.tensor(VALUES)[:, None].expand(len(VALUES), width).contiguous()


def most(x):
    """|hat| at most.  The first mean is off by DEPTH roundings of it, so is the mean of what it leaves, relative to that; what
    both leave is divided by sqrt(eps), and a rounding of each step along."""
    off = 1.1 * DEPTH * U32
    return ((off * off + 4 * U32 * off) * np.abs(f64(x)) + 2.0 ** -140) / np.sqrt(EPS)


@pytest.mark.parametrize("width", WIDTHS)
def test_they_come_out_as_the_bias(width):
    x = rows(width)
    params = torch.randn(2 * width, generator=torch.Generator().manual_seed(width))
    bias, weight = f64(params[:width]), f64(params[width:])
    form = dict(eps=EPS, norm="layer")
    y = B.adasum_join(B.Join(width, torch.float32, before_bias=0, before_weight=width, **form), params.cuda(), x.cuda(), keep_h=False)[1]
    h, _ = B.adasum_join(B.Join(width, torch.float32, after=True, before=False, after_bias=0, after_weight=width, **form), params.cuda(), x.cuda())
    for got in (y, h):
        assert (np.abs(f64(got) - bias) <= most(x) * np.abs(weight) + U32 * np.abs(bias)).all()


@pytest.mark.parametrize("width", WIDTHS[1:])
def test_their_gradient(width):
    """hat is 0: one over sqrt(eps) times what is left of dy without its mean; the weight's gradient is 0, the bias's sum_t dy."""
    x = rows(width)
    dy = torch.randn(len(VALUES), width, generator=torch.Generator().manual_seed(width))
    grad = torch.zeros(2 * width, device="cuda")
    dx, _ = B.adasum_join_grad(B.Join(width, torch.float32, before_bias=0, before_weight=width, eps=EPS), torch.ones(2 * width, device="cuda"), grad,
                               h=x.cuda(), dy=dy.cuda(), dresidual=False)
    d, hat = f64(dy), most(x)
    size = np.abs(d) + np.abs(d).mean(1, keepdims=True)
    # sums of a row and some ten steps more; of the spread, and of hat times the mean of dy hat, what a hat of that size leaves
    tol = (U32 * (DEPTH + 10) + hat * hat) * size / np.sqrt(EPS)
    assert (np.abs(f64(dx) - (d - d.mean(1, keepdims=True)) / np.sqrt(EPS)) <= tol).all()
    assert (np.abs(f64(grad[width:])) <= (np.abs(d) * hat).sum(0) * 1.01).all()
    assert (np.abs(f64(grad[:width]) - d.sum(0)) <= 8 * U32 * np.abs(d).sum(0)).all()


def test_a_small_spread_beside_a_large_mean():
    """Whole numbers around 4096 in fp32: the mean's own remainder counts, the values are exact."""
    width = 1000
    x = 4096.0 + torch.randint(-1, 2, (50, width), generator=torch.Generator().manual_seed(1)) * 2.0 ** -11
    y = B.adasum_join(B.Join(width, torch.float32, eps=EPS), None, x.cuda(), keep_h=False)[1]
    t = f64(x)
    t = t - t.mean(1, keepdims=True)
    spread = np.sqrt((t * t).mean(1, keepdims=True) + EPS)
    # the first mean is off by DEPTH roundings of 4096, the second by as many of what the first leaves, on top of values as large as the
    # spread (whose mean size is at most that); the spread by as many of itself
    off = 1.1 * DEPTH * U32
    assert (np.abs(f64(y) - t / spread) <= off * off * 4096 / spread + (DEPTH + 10) * U32 * (1 + np.abs(t / spread))).all()


@pytest.mark.parametrize("width", WIDTHS[1:])
def test_other_rows_do_not_notice(width):
    """The same bits for ordinary rows, whatever the rows beside them in a wave or a workgroup are."""
    g = torch.Generator().manual_seed(width)
    x, dy = torch.randn(70, width, generator=g), torch.randn(70, width, generator=g)
    mixed = x.clone()
    mixed[::3] = 100.3
    mixed[1::6] += 4000.0
    rest = [i for i in range(70) if i % 3 and i % 6 != 1]
    form = B.Join(width, torch.float32, eps=EPS)
    out = []
    for t in (x, mixed):
        y = B.adasum_join(form, None, t.cuda(), keep_h=False)[1]
        out.append((y, B.adasum_join_grad(form, None, None, h=t.cuda(), dy=dy.cuda(), dresidual=False)[0]))
    for a, b in zip(*out):
        assert torch.equal(a[rest], b[rest])
