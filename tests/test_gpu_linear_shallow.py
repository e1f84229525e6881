"""Products of at most 128 in depth with 16-bit results, by tiles of 64: of more than 4096 tiles of 16 x 16, in at most 128 tiles of edge 128."""
import numpy as np
import pytest
import torch

from between_util import in_8_bits
from layer_grads_util import f64
from paper_2006_02924_amd import binding as B
from test_gpu_linear_products import bound, near, spread

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
SIZES = [(2048, 128, 1024), (2000, 100, 1000), (4093, 64, 500), (16384, 128, 128), (16300, 60, 120), (500, 64, 4090), (1568, 128, 1000), (2048, 7, 1024),
         (1985, 1, 1021), (1100, 100, 1000), (1088, 128, 1024), (8800, 33, 120)]                         # rows, depth, results of a row
GUARD = 77.0


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def by_tiles_of_64(n, depth, there, out):
    """Whether the sizes are what this file is about: the workspace has both operands' values, and there are few tiles of 128."""
    need = B.adasum_linear_workspace_bytes(n, depth, there, out)
    return need >= (n + there) * 128 * 2 and -(-n // 128) * -(-there // 128) <= 128


def guarded(n, there, gap, dtype):
    """(rows to write to, the whole that they lie in): gaps between the rows, and more rows behind the last."""
    whole = torch.full((n + 40, there + gap), GUARD, dtype=dtype, device="cuda")
    return whole[:n, :there], whole


def untouched(whole, n, there):
    return bool((whole[n:] == GUARD).all()) and bool((whole[:n, there:] == GUARD).all())


def weights(backward, values, depth, there):
    """A layer whose forward product, or whose input's gradient, has this depth and these results: values [there][depth]."""
    w = values.t().contiguous() if backward else values
    return B.adasum_linear_store(w.reshape(-1).cuda(), 0, *w.shape)


def product(backward, weight, x, to):
    return B.adasum_linear_grad(weight, x, out=to) if backward else B.adasum_linear(weight, x, out=to)


@pytest.mark.parametrize("out", TYPES, ids=str)
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("n, depth, there", SIZES)
@pytest.mark.parametrize("gap", [0, 24, 5])
def test_whole_numbers(n, depth, there, backward, out, gap):
    """Sums that every type holds; nothing beside the result is written.  (The gap of 0 leaves the rows behind the last for the stores that would
    go past it.)"""
    assert by_tiles_of_64(n, depth, there, out)
    g = torch.Generator().manual_seed(depth)
    w, x = (torch.randint(-1, 2, shape, generator=g).float() for shape in ((there, depth), (n, depth)))
    weight = weights(backward, w, depth, there)
    to, whole = guarded(n, there, gap, out)
    assert torch.equal(product(backward, weight, x.cuda(), to).cpu().double(), x.double() @ w.double().t())
    assert untouched(whole, n, there)


@pytest.mark.parametrize("out", TYPES, ids=str)
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("n, depth, there", SIZES[:5])
def test_values(n, depth, there, backward, out):
    """The operands are multiplied as bf16 numbers, which hold them: sums in fp32, rounded once."""
    w = rand(1, there, depth) * 0.1
    x = spread(2, n, depth, torch.bfloat16).clamp(-60, 60)
    weight = weights(backward, w, depth, there)
    # (a weight's block of 128 x 128 is the same block of its transpose)
    w8, x8 = in_8_bits(f64(w), 128)[0], in_8_bits(f64(x), 1)[0]
    to, whole = guarded(n, there, 3, out)
    near(product(backward, weight, x.cuda(), to), x8 @ w8.T, bound(x8, w8, depth, torch.float32))
    assert untouched(whole, n, there)


@pytest.mark.parametrize("out", TYPES, ids=str)
def test_with_a_bias(out):
    n, depth, there = 2000, 100, 1000
    g = torch.Generator().manual_seed(3)
    w, x, b = (torch.randint(-1, 2, shape, generator=g).float() for shape in ((there, depth), (n, depth), (there,)))
    flat = torch.cat([w.reshape(-1), b]).cuda()
    weight = B.adasum_linear_store(flat, 0, there, depth)
    to, whole = guarded(n, there, 8, out)
    B.adasum_linear(weight, x.to(out).cuda(), params=flat, bias_offset=there * depth, out=to)
    assert np.array_equal(f64(to), f64(x) @ f64(w).T + f64(b)) and untouched(whole, n, there)
