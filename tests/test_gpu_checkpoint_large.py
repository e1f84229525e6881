"""Checkpoints of many rows, of whole, ragged and short rows, and every activation's gradient from them, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from layer_grads_util import DTYPES, f64, half_step, keep, least, slope, split, values, within
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
SHAPES = [(17000, 1000, 8), (16500, 1001, 3), (530001, 5, 1), (66000, 256, 0)]


def some_activations(n, width, dtype):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, width, generator=g) * torch.exp2(torch.randint(-9, 5, (n, 1), generator=g).float())
    x[n // 2] = 0.0
    x[1, 0], x[n - 1, width - 1], x[n // 3, width // 2] = float("inf"), float("nan"), 60000.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, width, gap", SHAPES)
def test_store_load_and_every_activation(n, width, gap, dtype):
    # eight channels a lane: so many of them that every form for 16 bits that takes four at a time is reached; fp32 has no such form
    n = n // 8 if dtype == "f32" else n
    assert dtype == "f32" or n * (-(-width // 32) * 4) > 1 << 21
    dtype = DTYPES[dtype]
    x = torch.full((n, width + gap), float("nan"), dtype=dtype, device="cuda")
    given = some_activations(n, width, dtype)
    x[:, :width] = given.cuda()
    kept = B.adasum_checkpoint_store(x[:, :width])
    q, e = keep(f64(given))
    got_q, got_e = split(kept.data, n, width)
    assert np.array_equal(got_q, q) and np.array_equal(got_e, e)
    v = values(q, e, width)
    wide = torch.full((n, width + gap), 3.0, dtype=dtype, device="cuda")
    B.adasum_checkpoint_load(kept, out=wide[:, :width])
    assert np.array_equal(f64(wide[:, :width]), v, equal_nan=True) and (wide[:, width:] == 3.0).all()
    dy = torch.full((n, width + gap), float("nan"), dtype=dtype, device="cuda")
    dy[:, :width] = torch.randn(n, width, generator=torch.Generator().manual_seed(n + 1)).cuda()
    d = f64(dy[:, :width])
    for act in B.ACTS:
        s, tol = slope(v, act)
        want, tol = d * s, np.abs(d) * tol
        got = B.adasum_checkpoint_act_grad(kept, dy[:, :width], act)
        within(f64(got), want, tol + (half_step(dtype) + 2.0 ** -24) * (np.abs(want) + tol) + least(dtype))
        wide.fill_(3.0)
        wide[:, :width] = dy[:, :width]
        B.adasum_checkpoint_act_grad(kept, wide[:, :width], act, out=wide[:, :width])            # in place
        assert torch.equal(wide[:, :width].nan_to_num(7.0), got.nan_to_num(7.0)) and (wide[:, width:] == 3.0).all()
