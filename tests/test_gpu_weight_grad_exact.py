"""Weight and bias gradients whose sums are exact: every element has one value, in every kind of square and split."""
import pytest
import torch

from layer_grads_util import DTYPES
from paper_2006_02924_amd import binding as B
from weight_grad_cases import CASES, gradients, inputs

pytestmark = pytest.mark.gpu


def check(case, kind, lead, gap, accumulate):
    out = DTYPES[case[1]]
    dy, x = inputs(case, kind, "cuda")
    n, outputs = dy.shape
    width = x.shape[1]
    kept = B.adasum_checkpoint_store(x)
    assert torch.equal(B.adasum_checkpoint_load(kept), x)
    wide = torch.full((n, outputs + gap), float("nan"), dtype=dy.dtype, device="cuda")
    wide[:, :outputs] = dy
    size = outputs * width
    flat = torch.full((lead + size + outputs + 9,), 5.0, dtype=out, device="cuda")
    old = flat[lead:lead + size + outputs]
    if accumulate:
        g = torch.Generator(device="cuda").manual_seed(2)
        old.copy_(torch.randint(-60, 60, old.shape, generator=g, device="cuda"))
    before = old.clone() if accumulate else torch.zeros_like(old)
    weight, bias = gradients(dy, x, before[:size].view(outputs, width), before[size:], out)
    B.adasum_checkpoint_weight_grad(kept, wide[:, :outputs], flat, lead, bias_offset=lead + size, accumulate=accumulate)
    assert torch.equal(old[:size].view(outputs, width), weight) and torch.equal(old[size:], bias)
    assert (flat[:lead] == 5).all() and (flat[lead + size + outputs:] == 5).all()


@pytest.mark.parametrize("accumulate", [False, True], ids=["over", "add"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_whole_numbers(case, accumulate):
    check(case, "whole", 3 if accumulate else 0, 0 if accumulate else 8, accumulate)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] == "f32"], ids=lambda c: "-".join(map(str, c)))
def test_numbers_of_three_parts(case):
    check(case, "three parts", 0, 0, False)
    check(case, "three parts", 5, 3, False)


def test_the_ends_of_fp32():
    """One token an output: its product is what is stored.  Values that bf16 would round to an infinity, powers of two, ties between bf16's
    numbers, and the least ones whose three parts bf16 holds."""
    f = torch.finfo(torch.float32)
    values = [f.max, -f.max, 3.3961775e38, 3.396e38, -3.39e38, 3.3895314e38, 2.0 ** 127, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -23,
              1 - 2.0 ** -24, 1 + 2.0 ** -7 - 2.0 ** -23, (2 - 2.0 ** -23) * 2.0 ** -110, (1 + 2.0 ** -23) * 2.0 ** -110, 0.0, -0.0]
    n = len(values)
    dy = torch.diag(torch.tensor(values, dtype=torch.float64)).float()
    x = torch.full((n, 32), 2.0 ** -3)
    x[:, ::2] = -7 * 2.0 ** -6
    kept = B.adasum_checkpoint_store(x.cuda())
    assert torch.equal(B.adasum_checkpoint_load(kept).cpu(), x)
    flat = torch.empty(n * 33, device="cuda")
    B.adasum_checkpoint_weight_grad(kept, dy.cuda(), flat, 0, bias_offset=n * 32)
    d = dy.double().sum(1)
    got, want = flat[:n * 32].view(n, 32).cpu().double(), d[:, None] * x.double()
    assert torch.equal(got[:, 1::2], want[:, 1::2])
    # seven times a value may need a rounding, and each part's product is added to what the parts before gave: two roundings of at most one step
    assert ((got - want).abs() <= 2 * 2.0 ** -23 * want.abs()).all()
    assert torch.equal(flat[n * 32:].cpu().double(), d)
