"""Long sums of one sign: the roundings of a weight's gradient go either way, in sums that one workgroup forms alone and in joined ones."""
import pytest
import torch

from layer_grads_util import DTYPES
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, outputs, width, joined", [(8192, 4096, 4096, False), (6000, 4095, 4096, False), (40000, 512, 1024, True)])
def test_roundings_of_long_sums_go_either_way(dtype, n, outputs, width, joined):
    dtype = DTYPES[dtype]
    assert (B.adasum_checkpoint_weight_grad_workspace_bytes(n, width, outputs, dtype) > 0) == joined
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.randn(n, width, generator=g, device="cuda").abs() + 0.5).to(dtype)
    dy = (torch.randn(n, outputs, generator=g, device="cuda").abs() + 0.5).to(dtype)
    kept = B.adasum_checkpoint_store(x)
    flat = torch.empty(outputs * (width + 1), device="cuda")
    B.adasum_checkpoint_weight_grad(kept, dy, flat, 0, bias_offset=outputs * width)
    d = dy.double()
    want = torch.matmul(d.t().contiguous(), B.adasum_checkpoint_load(kept).double())
    off = (flat[:outputs * width].view(outputs, width).double() / want - 1) * 2.0 ** 23        # in steps of fp32, or half of them
    # A matrix instruction adds sixteen products, with at most four roundings of half a step each: 4 * 3 * n / 16 of them for fp32's three
    # parts.  If each may go either way that is a walk of at most (3 n / 4 / 12)^0.5 = (n / 16)^0.5 steps, which no element of some
    # million exceeds eight times, and which cancels in the average over them.  Roundings that go one way add up to n / 16 half
    # steps at least; third parts that are lost, to 2^-17 of the sum, 64 steps.
    assert abs(float(off.mean())) < 1
    assert float(off.abs().max()) < 8 * (n / 16) ** 0.5 + 2
    # dy's sums: cut off in runs of a step's tokens, which 16 additions make (16 steps of the run at most), and rounded beyond
    off = (flat[outputs * width:].double() / d.sum(0) - 1) * 2.0 ** 23
    assert float(off.abs().max()) < 3 * 16 + 8 * (n / 32 / 12) ** 0.5 + 2
