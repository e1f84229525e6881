"""What the end of a join's sums makes of the gate's gradient when there is no bias to multiply the other sum with."""
import pytest
import torch

from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("after", [False, True])
def test_a_sum_beyond_the_range_that_nothing_asks_for(after):
    """sum_t D leaves the range of fp32, sum_t D x does not: without a bias behind the norm only the second one counts."""
    n, width = 4, 24
    x = torch.full((n, width), 2.0 ** -40)
    x[:, ::2] *= -1
    dh = torch.full((n, width), 2.0 ** 127)
    form = B.Join(width, torch.float32, norm="rms", eps=1.0, after=after, before=False, gate=0, after_weight=width if after else None)
    params = torch.ones(2 * width, device="cuda")
    grad = torch.zeros(2 * width, device="cuda")
    B.adasum_join_grad(form, params, grad, x=x.cuda(), dh=dh.cuda(), dresidual=False)
    want = x.double()      # (squares of 2^-40 beside an eps of 1: the normed rows are the rows)
    assert torch.equal(grad[:width].cpu().double(), (want * dh.double()).sum(0))
