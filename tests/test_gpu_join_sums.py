"""Sums of the parameters' gradients of a join: where fp32 ends and fp64 begins."""
import pytest
import torch

from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width, rows", [(8, 32), (64, 32), (100, 16), (130, 8), (256, 8), (257, 4), (512, 4), (1000, 4), (1024, 4)])
def test_rows_that_a_workgroup_has_at_once(width, rows):
    """One row of each lane: nothing is added up in fp32.  2^24 and ones, which fp32 would lose one by one."""
    dy = torch.ones(rows, width)
    dy[0] = 2.0 ** 24
    h = torch.randn(rows, width, generator=torch.Generator().manual_seed(1))
    grad = torch.zeros(width, device="cuda")
    B.adasum_join_grad(B.Join(width, torch.float32, before_bias=0), torch.zeros(width, device="cuda"), grad, h=h.cuda(), dy=dy.cuda(), dresidual=False)
    # rounded to fp32 (steps of 2 there) as the workgroup's sum, the only one
    assert (grad.cpu().double() - (2.0 ** 24 + rows - 1)).abs().max() <= 1.0
    gate, ones = torch.zeros(width, device="cuda"), torch.ones(rows, width, device="cuda")
    B.adasum_join_grad(B.Join(width, torch.float32, before=False, gate=0), torch.ones(width, device="cuda"), gate, x=ones, dh=dy.cuda(), dresidual=False)
    assert (gate.cpu().double() - (2.0 ** 24 + rows - 1)).abs().max() <= 1.0
