"""Activation checkpoints in 8 bits, and the gradient through an activation function from one, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from layer_grads_util import DTYPES, f64, half_step, keep, least, slope, split, values, within
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
KEPT = ["f32", "bf16", "f16"]


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def activations(seed, n, width, dtype):
    """Rows of many magnitudes, with zeros, ties, the type's largest and smallest values, infinities and NaN."""
    x = rand(seed, n, width) * torch.exp2(torch.randint(-30 if dtype != torch.float16 else -10, 11, (n, 1),
                                                        generator=torch.Generator().manual_seed(seed + 1)).float())
    x = x.to(dtype)
    f = torch.finfo(dtype)
    special = [0.0, f.max, -f.max, f.smallest_normal, f.smallest_normal * f.eps, float("inf"), float("nan"), float("-inf"), 127.5, 127.75]
    for i, v in enumerate(special):
        if n > i + 1:
            x[i + 1, (7 * i) % width] = v
    if n > 20:
        x[12] = 0.0
        x[13] = f.smallest_normal * f.eps
        x[14] = (torch.arange(width) % 128).to(dtype) + 0.5       # ties
        x[15] = f.max
        x[16] = (torch.arange(width) % 256).to(dtype) / 2 - 64
        x[17] = float("nan")
        x[18] = 1e-38 if dtype != torch.float16 else 1e-7
    return x


@pytest.mark.parametrize("dtype", KEPT)
@pytest.mark.parametrize("n, width, gap", [(1, 1, 0), (1, 32, 0), (3, 31, 2), (40, 33, 0), (30, 1023, 1), (64, 256, 8), (37, 4096, 0), (700, 520, 3)])
def test_store_and_load(dtype, n, width, gap):
    dtype = DTYPES[dtype]
    x = torch.full((n, width + gap), float("nan"), dtype=dtype)     # what lies between the rows is not looked at
    x[:, :width] = activations(n + width, n, width, dtype)
    dev = x.cuda()[:, :width]
    kept = B.adasum_checkpoint_store(dev)
    assert (kept.rows, kept.width, kept.dtype) == (n, width, dtype)
    q, e = keep(f64(x[:, :width]))
    got_q, got_e = split(kept.data, n, width)
    assert np.array_equal(got_q, q) and np.array_equal(got_e, e)
    want = values(q, e, width)
    assert np.array_equal(f64(B.adasum_checkpoint_load(kept)), want, equal_nan=True)      # exact in the type that x had
    wide = torch.full((n, width + gap), 3.0, device="cuda")
    B.adasum_checkpoint_load(kept, out=wide[:, :width])
    assert np.array_equal(f64(wide[:, :width]), want, equal_nan=True) and (wide[:, width:] == 3.0).all()
    # how far it is from what was given: half a step of the block, a whole one beyond 127.5 steps
    fine = np.isfinite(want)
    step = np.ldexp(1.0, np.repeat(np.where(e == -128, 0, e), 32, axis=1)[:, :width].astype(int))
    off, given = np.abs(want - f64(x[:, :width])), np.abs(f64(x[:, :width]))
    assert (off[fine] <= np.where(given > 127.5 * step, 1.0, 0.5)[fine] * step[fine]).all()
    # what is kept is kept as it is a second time
    again = B.adasum_checkpoint_store(B.adasum_checkpoint_load(kept))
    assert np.array_equal(f64(B.adasum_checkpoint_load(again)), want, equal_nan=True)


@pytest.mark.parametrize("act", list(B.ACTS))
@pytest.mark.parametrize("dtype", KEPT)
@pytest.mark.parametrize("n, width, gap", [(1, 1, 0), (5, 33, 1), (40, 1000, 8), (300, 4096, 0)])
def test_gradient_through_an_activation(act, dtype, n, width, gap):
    dtype = DTYPES[dtype]
    x = rand(n, n, width) * 3
    x[n // 2] = torch.linspace(-40, 40, width) if width > 1 else -12.0
    if n > 4:
        x[0] = torch.linspace(-1, 1, width)
        x[1, 0] = float("nan")
        x[2] = 0.0
        x[3, :] = 60000.0
        x[4, :] = -60000.0
    kept = B.adasum_checkpoint_store(x.to(dtype).cuda())
    dy = torch.full((n, width + gap), float("nan"), dtype=dtype)
    dy[:, :width] = rand(n + 1, n, width).to(dtype)
    dev = dy.cuda()[:, :width]
    s, tol = slope(f64(B.adasum_checkpoint_load(kept)), act)
    d = f64(dev)
    want = d * s
    tol = np.abs(d) * tol
    tol = tol + (half_step(dtype) + 2.0 ** -24) * (np.abs(want) + tol) + least(dtype)
    got = B.adasum_checkpoint_act_grad(kept, dev, act)
    within(f64(got), want, tol)
    wide = torch.full((n, width + gap), 3.0, dtype=dtype, device="cuda")
    wide[:, :width] = dev
    assert B.adasum_checkpoint_act_grad(kept, wide[:, :width], act, out=wide[:, :width]) is not None     # in place
    assert torch.equal(wide[:, :width].nan_to_num(7.0), got.nan_to_num(7.0)) and (wide[:, width:] == 3.0).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_slope_against_differences(act):
    """dy = 1 gives the slope: the difference quotient of the function itself at the kept values."""
    x = torch.linspace(-9, 9, 4096)[None]
    kept = B.adasum_checkpoint_store(x.cuda())
    got = f64(B.adasum_checkpoint_act_grad(kept, torch.ones(1, 4096, device="cuda"), act))[0]
    v = B.adasum_checkpoint_load(kept).cpu().double()[0]
    fn = {"gelu": lambda t: torch.nn.functional.gelu(t), "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh"),
          "silu": torch.nn.functional.silu}[act]
    h = 2.0 ** -16
    want = ((fn(v + h) - fn(v - h)) / (2 * h)).numpy()
    # third derivative below 2, h^2 / 6 of it; rounding of values below 9; fp32 of the slope, whose argument's share stays below 2^-17 here
    assert np.abs(got - want).max() < 2 * h * h / 6 + 9 * 2.0 ** -52 / h + 2.0 ** -17


def test_rows_beyond_32_bits():
    n, width = (1 << 20) + 3, 2080
    x = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    x[n - 1] = torch.linspace(-3, 3, width, device="cuda")
    x[0] = 1.0
    kept = B.adasum_checkpoint_store(x)
    back = B.adasum_checkpoint_load(kept)
    want = values(*keep(f64(x[n - 1:])), width)
    assert np.array_equal(f64(back[n - 1:]), want) and (back[0] == 1.0).all() and int(torch.count_nonzero(back[1:n - 1])) == 0
    got = B.adasum_checkpoint_act_grad(kept, x, "relu")
    assert np.array_equal(f64(got[n - 1:]), f64(x[n - 1:]) * (want > 0)) and (got[0] == 1.0).all()


def test_captured_and_on_another_stream():
    x, dy = rand(1, 500, 1000).bfloat16().cuda(), rand(2, 500, 1000).bfloat16().cuda()
    kept = B.Checkpoint(500, 1000, torch.bfloat16, device="cuda")
    out, dx = torch.empty_like(x), torch.empty_like(x)

    def all_three(**kw):
        B.adasum_checkpoint_store(x, out=kept, **kw)
        B.adasum_checkpoint_load(kept, out=out, **kw)
        B.adasum_checkpoint_act_grad(kept, dy, "gelu", out=dx, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    all_three(stream=side)
    side.synchronize()
    first = out.clone(), dx.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_three()
    for rep in range(3):
        x.copy_(rand(10 + rep, 500, 1000))
        again = B.adasum_checkpoint_store(x)
        want = B.adasum_checkpoint_load(again), B.adasum_checkpoint_act_grad(again, dy, "gelu")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(dx, want[1]) and not torch.equal(out, first[0])


def test_the_binding_refuses_wrong_shapes():
    x = torch.zeros(4, 40, device="cuda")
    kept = B.adasum_checkpoint_store(x)
    for bad in (lambda: B.adasum_checkpoint_store(x.t()), lambda: B.adasum_checkpoint_store(x[:3], out=kept),
                lambda: B.adasum_checkpoint_store(x.half(), out=kept), lambda: B.adasum_checkpoint_load(kept, out=x[:3]),
                lambda: B.adasum_checkpoint_load(kept, out=x.cpu()), lambda: B.adasum_checkpoint_act_grad(kept, x[:, :39], "gelu"),
                lambda: B.adasum_checkpoint_act_grad(kept, x, "gelu", out=x.half()), lambda: B.adasum_checkpoint_store(x[0])):
        with pytest.raises(ValueError):
            bad()
