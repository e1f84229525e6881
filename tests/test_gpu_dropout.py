"""Dropout whose mask is never stored, bit by bit against its definition."""
import numpy as np
import pytest
import torch

from between_util import kept, philox
from layer_grads_util import DTYPES
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
KEPT = ["f32", "bf16", "f16"]
SEED = 0x9ABCDEF012345678


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def defined(x, p, seed, step=0):
    """The product in fp32, rounded once more to the type; nothing else is rounded."""
    mask, factor = kept(x.shape[0], x.shape[1], p, seed, step)
    return torch.where(torch.from_numpy(mask), x.float() * torch.tensor(factor, dtype=torch.float32), torch.zeros(())).to(x.dtype)


@pytest.mark.parametrize("dtype", KEPT)
@pytest.mark.parametrize("n, width, gap", [(1, 1, 0), (1, 8, 0), (3, 7, 2), (40, 33, 1), (30, 1023, 0), (64, 256, 8), (9, 4096, 0), (700, 520, 3), (1200, 4096, 0)])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_values(dtype, n, width, gap, p):
    dtype = DTYPES[dtype]
    x = torch.full((n, width + gap), float("nan"), dtype=dtype)
    x[:, :width] = rand(n + width, n, width).to(dtype)
    dev = x.cuda()[:, :width]
    step = torch.tensor([5 + (3 << 40)], dtype=torch.int64, device="cuda")
    want = defined(x[:, :width], p, SEED, int(step))
    wide = torch.full((n, width + gap), 3.0, dtype=dtype, device="cuda")
    B.adasum_dropout(dev, p, SEED, step=step, out=wide[:, :width])
    assert torch.equal(wide[:, :width].cpu(), want) and (wide[:, width:] == 3.0).all()
    assert torch.equal(B.adasum_dropout(dev, p, SEED).cpu(), defined(x[:, :width], p, SEED))
    # in place, between the rows' gaps
    B.adasum_dropout(dev, p, SEED, step=step, out=dev)
    assert torch.equal(dev.cpu(), want)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.9, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1.0])
def test_shares_at_the_ends(p):
    x = rand(1, 50, 300)
    assert torch.equal(B.adasum_dropout(x.cuda(), p, 77).cpu(), defined(x, p, 77))


def test_dropped_places_are_zero_whatever_they_hold():
    x = torch.full((20, 100), float("nan"))
    x[10:] = float("inf")
    got = B.adasum_dropout(x.cuda(), 0.5, 3).cpu()
    mask, _ = kept(20, 100, 0.5, 3)
    mask = torch.from_numpy(mask)
    assert (got[~mask] == 0).all() and got[:10][mask[:10]].isnan().all() and got[10:][mask[10:]].isinf().all()


def test_more_dimensions_and_shared_rows():
    x = rand(2, 6, 5, 40).bfloat16()
    assert torch.equal(B.adasum_dropout(x.cuda(), 0.3, 9).cpu().view(30, 40), defined(x.view(30, 40), 0.3, 9))
    one = x[0, :1].cuda().expand(30, 40)
    assert torch.equal(B.adasum_dropout(one, 0.3, 9, out=torch.empty(30, 40, dtype=torch.bfloat16, device="cuda")).cpu(), defined(one.cpu(), 0.3, 9))


def test_rows_beyond_32_bits():
    n, width = (1 << 20) + 3, 2080
    x = torch.ones(n, width, dtype=torch.bfloat16, device="cuda")
    got = B.adasum_dropout(x, 0.5, SEED)
    granules = np.arange(width // 8)
    for row in (0, 1, n // 2, n - 2, n - 1):
        words = philox([granules, np.full_like(granules, row), 0 * granules, 0 * granules], [SEED % 2 ** 32, SEED >> 32])
        halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)
        assert np.array_equal(got[row].float().cpu().numpy(), np.where(halves >= 32768, 2.0, 0.0))
    # five deviations of as many draws
    assert abs(float((got != 0).double().mean()) - 0.5) < 5 * 0.5 / (n * width) ** 0.5


def test_captured_with_a_step_that_moves():
    x = rand(4, 300, 512).bfloat16().cuda()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.adasum_dropout(x, 0.2, SEED, step=step, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out.cpu(), defined(x.cpu(), 0.2, SEED))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adasum_dropout(x, 0.2, SEED, step=step, out=out)
        step.add_(1)
    for rep in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == rep + 1 and torch.equal(out.cpu(), defined(x.cpu(), 0.2, SEED, rep)), rep


def test_refusals():
    x = torch.zeros(4, 40, device="cuda")
    step = torch.zeros(2, dtype=torch.int64, device="cuda")
    for bad in (lambda: B.adasum_dropout(x, 0.1, 1, step=step), lambda: B.adasum_dropout(x, 0.1, 1, step=step[:1].cpu()),
                lambda: B.adasum_dropout(x, 0.1, 1, step=step[:1].int()), lambda: B.adasum_dropout(x, 0.1, 1, out=x[:3]),
                lambda: B.adasum_dropout(x, 0.1, 1, out=x.half()), lambda: B.adasum_dropout(x.t(), 0.1, 1), lambda: B.adasum_dropout(x[0], 0.1, 1)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.AdasumError):
        B.adasum_dropout(x, 1.5, 1)
    assert B.adasum_dropout(x[:0], 0.1, 1).shape == (0, 40)
    assert torch.equal(B.adasum_dropout(x, 0.1, 1, step=step[1:]), x)      # a step at eight bytes of sixteen
