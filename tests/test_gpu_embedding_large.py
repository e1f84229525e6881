"""Many tokens: rows looked up and the table's gradient with sums that are exact, so that every element has one value."""
import pytest
import torch

from layer_grads_util import DTYPES, PAIRS
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


def some_ids(n, rows, seed):
    """A few rows that many tokens name, many that few or none do, one in seven no row at all."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) ** 3 * rows).long()
    none = torch.rand(n, generator=g, device="cuda") < 1 / 7
    ids[none] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1, rows)[none]
    return ids


# tokens, rows, width, type of dy and of the gradient, offset, gap.  Beyond 32768 tokens chunks are of 32; sorted by two launches up to 262144
# rows, where ranges of one row (up to 256 rows) go another way, and by one beyond; rows of whole granules, ragged and short ones.
GRADS = [(40000, 5000, 104, "bf16", "f32", 3, 0), (33000, 3001, 1023, "f32", "bf16", 1, 5), (70001, 7919, 520, "f16", "f16", 0, 8),
         (40000, 1000, 3, "f32", "f32", 7, 2), (50000, 4099, 65, "f64", "f64", 1, 0), (40000, 300001, 9, "bf16", "bf16", 5, 1),
         (36000, 262145, 16, "f32", "f16", 0, 0), (65501, 2, 1001, "bf16", "f32", 1, 3), (65501, 256, 70, "f16", "bf16", 0, 0),
         (40000, 257, 12, "bf16", "f16", 0, 4), (32768, 5000, 65, "f16", "f32", 0, 0), (32769, 5000, 65, "f16", "f32", 0, 0),
         (131072, 30522, 64, "f32", "f32", 9, 0), (90000, 40000, 5, "bf16", "bf16", 2, 0)]


@pytest.mark.parametrize("n, rows, width, dtype, out, offset, gap", GRADS)
def test_table_gradient(n, rows, width, dtype, out, offset, gap):
    dtype, out = DTYPES[dtype], DTYPES[out]
    g = torch.Generator(device="cuda").manual_seed(n)
    wide = torch.full((n, width + gap), float("nan"), dtype=dtype, device="cuda")
    dy = wide[:, :width]
    dy.copy_(torch.randint(-8, 9, (n, width), generator=g, device="cuda"))
    ids = some_ids(n, rows, n + 1)
    there = (ids >= 0) & (ids < rows)
    sums = torch.zeros(rows, width, dtype=torch.float64, device="cuda").index_add_(0, ids[there], dy[there].double())
    dy[~there] = float("inf")                                  # what padding carries is not looked at
    flat = torch.full((offset + rows * width + 9,), 5.0, dtype=out, device="cuda")
    layer = flat[offset:offset + rows * width].view(rows, width)
    B.adasum_embedding_grad(dy, ids, flat, offset, rows, scale=0.5)
    assert torch.equal(layer, (sums * 0.5).to(out))
    # added to what is there, by ids of 32 bits
    old = torch.randint(-30, 31, (rows, width), generator=g, device="cuda").to(out)
    layer.copy_(old)
    B.adasum_embedding_grad(dy, ids.int(), flat, offset, rows, scale=0.5, accumulate=True)
    assert torch.equal(layer, (sums * 0.5 + old.double()).to(out))
    assert (flat[:offset] == 5).all() and (flat[offset + rows * width:] == 5).all()


@pytest.mark.parametrize("dtype, out", PAIRS)
@pytest.mark.parametrize("n, rows, width, offset, gap", [(40000, 30522, 104, 8, 0), (33001, 2000, 77, 3, 5), (300001, 500, 3, 1, 1)])
def test_lookup(dtype, out, n, rows, width, offset, gap):
    dtype, out = DTYPES[dtype], DTYPES[out]
    g = torch.Generator(device="cuda").manual_seed(width)
    params = (torch.randn(offset + rows * width + 3, generator=g, device="cuda") * 3).to(dtype)
    ids = some_ids(n, rows, n)
    wide = torch.full((n, width + gap), 7.0, dtype=out, device="cuda")
    B.adasum_embedding(params, offset, rows, width, ids, scale=4.0, out=wide[:, :width])
    table = params[offset:offset + rows * width].view(rows, width)
    want = (table[ids.clamp(0, rows - 1)] * 4.0 if dtype == torch.float64 else table[ids.clamp(0, rows - 1)].float() * 4.0).to(out)
    want[(ids < 0) | (ids >= rows)] = 0
    assert torch.equal(wide[:, :width], want) and (wide[:, width:] == 7).all()
