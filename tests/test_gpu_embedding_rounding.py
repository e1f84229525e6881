"""The table's gradient is rounded once: long runs of tokens, whose sums are formed in fp64, into 16-bit gradients."""
import pytest
import torch

from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


def sums_of(column, dtype, old):
    """The gradient of two rows of one element; row 1's tokens carry `column`, 300 tokens that no chunk holds alone."""
    n = 300
    dy = torch.zeros(n, 1)
    for place, value in column.items():
        dy[place] = value
    grad = torch.full((2,), old, dtype=dtype, device="cuda")
    B.adasum_embedding_grad(dy.cuda(), torch.ones(n, dtype=torch.int32, device="cuda"), grad, 0, 2, accumulate=old != 0)
    assert grad[0].item() == old
    return grad[1].item()


# (what lies half way between two numbers of the type, what decides it, the result)
HALF_WAY = {
    torch.bfloat16: [(1 + 2.0 ** -8, 2.0 ** -30, 1 + 2.0 ** -7), (1 + 2.0 ** -8, -2.0 ** -30, 1.0), (1 + 3 * 2.0 ** -8, -2.0 ** -30, 1 + 2.0 ** -7),
                     (-1 - 2.0 ** -8, -2.0 ** -30, -1 - 2.0 ** -7), (1 + 2.0 ** -8, 0.0, 1.0), (1 + 3 * 2.0 ** -8, 0.0, 1 + 2.0 ** -6),
                     ((2 - 2.0 ** -8) * 2.0 ** 127, -2.0 ** 90, (2 - 2.0 ** -7) * 2.0 ** 127), ((2 - 2.0 ** -8) * 2.0 ** 127, 0.0, float("inf"))],
    torch.float16: [(1 + 2.0 ** -11, 2.0 ** -40, 1 + 2.0 ** -10), (1 + 3 * 2.0 ** -11, -2.0 ** -40, 1 + 2.0 ** -10), (2.0 ** -25, 2.0 ** -60, 2.0 ** -24),
                    (3 * 2.0 ** -25, -2.0 ** -60, 2.0 ** -24), (-2.0 ** -25, 0.0, 0.0), (65520.0, -2.0 ** -20, 65504.0), (65520.0, 0.0, float("inf")),
                    (-65520.0, 2.0 ** -20, -65504.0), (2.0 ** 127, 2.0 ** 127, float("inf"))],
}


@pytest.mark.parametrize("dtype", list(HALF_WAY), ids=["bf16", "f16"])
def test_long_runs_are_rounded_once(dtype):
    for half, rest, want in HALF_WAY[dtype]:
        assert sums_of({3: half, 250: rest}, dtype, 0) == want, (half, rest)


@pytest.mark.parametrize("dtype, eps", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)], ids=["bf16", "f16"])
def test_long_runs_are_rounded_once_behind_what_is_added_to(dtype, eps):
    """1 and half of a step more: what is a little above goes up, what is a little below goes down."""
    for rest, want in ((2.0 ** -40, 1 + 2 * eps), (0.0, 1.0), (-2.0 ** -40, 1.0)):
        assert sums_of({0: eps, 299: rest}, dtype, 1.0) == want, rest


def test_infinities_and_nan_of_long_runs():
    inf = float("inf")
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        assert sums_of({7: inf}, dtype, 0) == inf and sums_of({7: -inf, 200: 1.0}, dtype, 0) == -inf
        nan = sums_of({7: inf, 200: -inf}, dtype, 0)
        assert nan != nan
