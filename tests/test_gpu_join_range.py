"""Norms of rows at the ends of the range: squares beyond fp32."""
import pytest
import torch

from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
WIDTHS = [7, 64, 200, 500, 1000, 2048, 4100, 8192]      # every count of lanes


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("width", WIDTHS)
def test_squares_beyond_the_range_give_no_numbers(width, dtype, norm):
    """1e20 squared is no fp32 number: the row is none either, in results and gradients; the rows beside it are what they are without it."""
    n, bad = 9, [2, 5]
    rest = [i for i in range(n) if i not in bad]
    params = rand(1, 2 * width).cuda()
    dy = rand(3, n, width).to(dtype).cuda()
    x = rand(2, n, width).to(dtype).cuda()
    dirty = x.clone()
    dirty[2], dirty[5, width // 2] = x[2] * 1e20, 3e20
    before = B.Join(width, dtype, norm=norm, before_weight=0, before_bias=width)
    clean, got = (B.adasum_join(before, params, t, keep_h=False)[1] for t in (x, dirty))
    assert torch.equal(got[rest], clean[rest]) and bool(got[bad].isnan().all())
    clean, got = (B.adasum_join_grad(before, params, torch.zeros_like(params), h=t, dy=dy, dresidual=False)[0] for t in (x, dirty))
    assert torch.equal(got[rest], clean[rest]) and bool(got[bad].isnan().all())
    # the norm after a block
    after = B.Join(width, dtype, norm=norm, after=True, before=False, after_weight=0, after_bias=width)
    clean, got = (B.adasum_join(after, params, t)[0] for t in (x, dirty))
    assert torch.equal(got[rest], clean[rest]) and bool(got[bad].isnan().all())
    clean, got = (B.adasum_join_grad(after, params, torch.zeros_like(params), x=t, dh=dy, dresidual=False)[0] for t in (x, dirty))
    assert torch.equal(got[rest], clean[rest]) and bool(got[bad].isnan().all())


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_squares_inside_the_range_are_numbers(norm):
    """Sums just inside it: 1000 squares of 2^58 are 2^126."""
    x = torch.where(rand(5, 4, 1000) < 0, -1.0, 1.0) * 2.0 ** 58
    y = B.adasum_join(B.Join(1000, torch.float32, norm=norm), None, x.cuda(), keep_h=False)[1]
    want = x.double() - (x.double().mean(1, keepdim=True) if norm == "layer" else 0.0)
    want = want / want.square().mean(1, keepdim=True).sqrt()
    # sums of 1000 terms in a tree and a few roundings: some 40 of 2^-24, of values near 1
    assert (y.cpu().double() - want).abs().max() < 50 * 2.0 ** -24
