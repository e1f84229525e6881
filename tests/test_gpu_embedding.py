"""Rows of an embedding table in a flat buffer and the table's gradient, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from layer_grads_util import DTYPES, PAIRS, f64, half_step, lane_u, least, within
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu


def rand(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * scale


def make_ids(seed, n, rows, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":            # all tokens name one row
        ids = torch.full((n,), rows // 2)
    elif kind == "few":          # long runs, their lengths around the length up to which a wave sums alone
        ids = torch.randint(0, max(1, min(rows, n // 33 + 1)), (n,), generator=g)
    elif kind == "distinct":
        ids = torch.arange(n) % rows
    else:
        ids = torch.randint(0, rows, (n,), generator=g)
    if kind == "padded" and n > 1:
        ids[torch.rand(n, generator=g) < 0.4] = -1
        ids[n // 2] = rows
        ids[n - 1] = 1 << 40
        ids[0] = -(1 << 40)
    return ids


def grad_reference(dy, ids, rows, scale, old=None):
    """The sums, and the sums of the magnitudes."""
    out, mag = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1]))
    for t, v in enumerate(ids.tolist()):
        if 0 <= v < rows:
            out[v] += dy[t]
            mag[v] += np.abs(dy[t])
    out, mag = out * scale, mag * abs(scale)
    return (out if old is None else out + old), mag


def check_grad(got, want, mag, dtype, out_dtype, old=None):
    # up to 32 rows are added in the lanes' type, such sums in fp64 (twice as much for fp64, whose reference is fp64 too); then the
    # factor, what was there, and the result's rounding
    u = lane_u(dtype) * (1 + (dtype == torch.float64) * 31)
    tol = 34 * u * mag + (half_step(out_dtype) + 2 * u) * np.abs(want) * (1 + 1e-6) + least(out_dtype)
    if old is not None:
        tol = tol + 2 * u * np.abs(old) + half_step(out_dtype) * 34 * u * mag
    within(got, want, tol)


@pytest.mark.parametrize("dtype, out", PAIRS)
@pytest.mark.parametrize("n, rows, width, offset, gap", [(1, 1, 1, 0, 0), (7, 5, 3, 1, 5), (64, 100, 64, 8, 0), (129, 33, 1000, 3, 8),
                                                         (300, 700, 1024, 0, 0), (5, 3, 4097, 2, 1)])
def test_lookup(dtype, out, n, rows, width, offset, gap):
    dtype, out = DTYPES[dtype], DTYPES[out]
    params = rand(1, offset + rows * width + 3).to(dtype).cuda()
    for kind, wide in (("any", True), ("padded", True), ("distinct", False)):
        ids = make_ids(2, n, rows, kind)
        dev = (ids if wide else ids.int()).cuda()
        wanted = torch.full((n, width + gap), 7.0, dtype=out, device="cuda")
        to = wanted[:, :width]
        assert B.adasum_embedding(params, offset, rows, width, dev, scale=1.7, out=to) is to
        table = f64(params)[offset:offset + rows * width].reshape(rows, width)
        there = ((ids >= 0) & (ids < rows)).numpy()
        factor = 1.7 if dtype == torch.float64 else float(np.float32(1.7))
        want = np.where(there[:, None], table[ids.clamp(0, rows - 1).numpy()] * factor, 0.0)
        u = lane_u(dtype)
        within(f64(to), want, (half_step(out) + u) * np.abs(want) * (1 + 1e-6) + least(out))
        assert (wanted[:, width:] == 7.0).all()


@pytest.mark.parametrize("dtype, out", PAIRS)
@pytest.mark.parametrize("n, rows, width, offset, gap, kind", [
    (1, 1, 1, 0, 0, "any"), (2, 5, 3, 1, 5, "any"), (33, 2, 8, 3, 0, "any"), (31, 40, 520, 0, 0, "distinct"), (32, 1, 16, 0, 1, "one"),
    (33, 1, 16, 5, 0, "one"), (64, 7, 24, 8, 8, "one"), (65, 3, 100, 1, 0, "few"), (500, 700, 1000, 7, 3, "padded"),
    (1000, 64, 130, 0, 0, "few"), (2111, 513, 64, 3, 0, "any"), (4097, 2, 40, 1, 0, "any"), (3000, 1200, 8, 0, 0, "few")])
def test_table_gradient(dtype, out, n, rows, width, offset, gap, kind):
    dtype, out = DTYPES[dtype], DTYPES[out]
    dy = torch.full((n, width + gap), float("nan"), dtype=dtype)
    dy[:, :width] = rand(3, n, width).to(dtype)
    ids = make_ids(n, n, rows, kind)
    if kind == "padded":      # what padding carries is not looked at
        dy[(ids < 0) | (ids >= rows)] = float("inf")
    dy_dev = dy.cuda()[:, :width]
    elems = rows * width
    flat = torch.full((offset + elems + 9,), 5.0, dtype=out, device="cuda")
    scale = float(np.float32(0.3))
    ids_dev = ids.cuda() if n % 2 else ids.clamp(-(1 << 31), (1 << 31) - 1).int().cuda()
    B.adasum_embedding_grad(dy_dev, ids_dev, flat, offset, rows, scale=scale)
    there = f64(torch.nan_to_num(dy[:, :width].double(), 0.0, 0.0, 0.0)) if kind == "padded" else f64(dy[:, :width])
    want, mag = grad_reference(there, ids, rows, scale)
    got = f64(flat)
    check_grad(got[offset:offset + elems].reshape(rows, width), want, mag, dtype, out)
    assert (got[:offset] == 5.0).all() and (got[offset + elems:] == 5.0).all()
    # added to what was there; rows that no token names stay as they are, bit for bit
    flat.copy_(rand(4, flat.numel()).to(out))
    before = f64(flat)
    old = before[offset:offset + elems].reshape(rows, width)
    B.adasum_embedding_grad(dy_dev, ids_dev, flat, offset, rows, scale=scale, accumulate=True)
    got = f64(flat)
    now = got[offset:offset + elems].reshape(rows, width)
    check_grad(now, want + old, mag, dtype, out, old)
    named = np.zeros(rows, dtype=bool)
    named[ids[(ids >= 0) & (ids < rows)].numpy()] = True
    assert np.array_equal(now[~named], old[~named])
    assert np.array_equal(got[:offset], before[:offset]) and np.array_equal(got[offset + elems:], before[offset + elems:])


def test_no_token_and_only_padding():
    flat = torch.ones(100, device="cuda")
    for ids in (torch.zeros(0, dtype=torch.int64), torch.full((50,), -1)):
        flat.fill_(1.0)
        dy = torch.full((ids.numel(), 8), float("nan"), device="cuda")
        B.adasum_embedding_grad(dy, ids.cuda(), flat, 4, 10, accumulate=True)
        assert (flat == 1.0).all()
        B.adasum_embedding_grad(dy, ids.cuda(), flat, 4, 10)
        assert (flat[4:84] == 0.0).all() and (flat[:4] == 1.0).all() and (flat[84:] == 1.0).all()
        out = B.adasum_embedding(flat, 0, 10, 8, ids.cuda())
        assert out.shape == (ids.numel(), 8) and (out == 0.0).all()


def test_infinities_and_nan_stay_in_their_row():
    dy = rand(5, 200, 64)
    ids = torch.arange(200) % 20
    dy[7] = float("inf")
    dy[28, 3] = float("nan")
    flat = torch.zeros(20 * 64, device="cuda")
    B.adasum_embedding_grad(dy.cuda(), ids.cuda(), flat, 0, 20)
    got = flat.view(20, 64).cpu()
    assert torch.isinf(got[7]).all() and torch.isnan(got[8, 3])
    got[7] = 0
    got[8, 3] = 0
    assert torch.isfinite(got).all()


def test_a_broadcast_gradient():
    """The gradient of a sum is one row, seen by every token (stride 0)."""
    one = rand(6, 1, 200).cuda()
    ids = make_ids(7, 3000, 50, "any")
    flat = torch.zeros(50 * 200, device="cuda")
    B.adasum_embedding_grad(one.expand(3000, 200), ids.cuda(), flat, 0, 50)
    counts = torch.bincount(ids, minlength=50).double()
    want = counts[:, None].numpy() * f64(one)
    check_grad(f64(flat).reshape(50, 200), want, np.abs(want), torch.float32, torch.float32)


def test_gradient_against_differences():
    """The lookup is linear: its directional derivative is the gradient's product with the direction."""
    rows, width, n = 30, 40, 100
    params = rand(8, rows * width).double().cuda()
    direction = rand(9, rows * width).double().cuda()
    ids = make_ids(10, n, rows, "padded").cuda()
    dy = rand(11, n, width).double().cuda()
    grad = torch.empty(rows * width, dtype=torch.float64, device="cuda")
    B.adasum_embedding_grad(dy, ids, grad, 0, rows, scale=3.0)
    h = 2.0 ** -10
    up, down = (B.adasum_embedding(params + s * h * direction, 0, rows, width, ids, scale=3.0) for s in (1, -1))
    slope = float(((up - down) * dy).sum()) / (2 * h)
    # 4000 products of size 3: rounding 2^-53 of values of a few units, divided by 2 h
    assert abs(slope - float((grad * direction).sum())) < 4000 * 3 * 32 * 2.0 ** -53 * 1024


@pytest.mark.parametrize("n, rows, width", [(50000, 30522, 256), (70001, 2, 1024), (20000, 140001, 8), (9000, 262144, 8), (20000, 300001, 8),
                                            (4096, 5000, 40), (4097, 5000, 40), (2200000, 300, 8), (30000, 1, 72), (8500000, 3, 1), (3000, 300001, 9)])
def test_larger_sums_are_right_and_the_same_every_time(n, rows, width):
    """More tokens than the sort takes at once, in every row or in a few, and tables on both sides of its limits."""
    g = torch.Generator().manual_seed(n)
    ids = (torch.rand(n, generator=g, dtype=torch.float64) ** 4 * rows).long()
    dy = torch.randn(n, width, generator=g).bfloat16()
    flat = torch.full((rows * width,), 9.0, device="cuda")
    dev, ids_dev = dy.cuda(), ids.cuda()
    B.adasum_embedding_grad(dev, ids_dev, flat, 0, rows)
    want = torch.zeros(rows, width, dtype=torch.float64).index_add_(0, ids, dy.double())
    mag = torch.zeros(rows, width, dtype=torch.float64).index_add_(0, ids, dy.double().abs())
    check_grad(f64(flat).reshape(rows, width), want.numpy(), mag.numpy(), torch.bfloat16, torch.float32)
    again = torch.full_like(flat, 3.0)
    B.adasum_embedding_grad(dev, ids_dev, again, 0, rows)
    assert torch.equal(flat, again)


def test_places_beyond_32_bits():
    """A table that lies, and goes on, beyond 2^31 elements of its flat buffer."""
    rows, width, offset = 1300000, 1024, (1 << 30) + 3
    flat = torch.ones(offset + rows * width + 5, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, rows - 1, 5, rows - 1, 1299998, -1]).cuda()
    dy = rand(12, 6, width).cuda()
    B.adasum_embedding_grad(dy, ids, flat, offset, rows)
    layer = flat[offset:offset + rows * width].view(rows, width)
    assert int(torch.count_nonzero(layer)) == int(sum(torch.count_nonzero(r) for r in (dy[0].bfloat16(), (dy[1] + dy[3]).bfloat16(), dy[2].bfloat16(),
                                                                                       dy[4].bfloat16())))
    assert torch.equal(layer[rows - 1], (dy[1] + dy[3]).bfloat16()) and torch.equal(layer[0], dy[0].bfloat16())
    assert torch.equal(layer[1299998], dy[4].bfloat16())
    assert (flat[:offset] == 1).all() and (flat[offset + rows * width:] == 1).all()
    out = B.adasum_embedding(flat, offset, rows, width, ids, out_dtype=torch.float32)
    assert torch.equal(out[1], layer[rows - 1].float()) and (out[5] == 0).all()


def test_captured_replayed_and_on_another_stream():
    rows, width, n = 1000, 256, 5000
    ids = make_ids(13, n, rows, "few").cuda()
    dy = rand(14, n, width).bfloat16().cuda()
    eager = torch.empty(rows * width, device="cuda")
    B.adasum_embedding_grad(dy, ids, eager, 0, rows)
    flat = torch.empty_like(eager)
    work = torch.empty(B.adasum_embedding_grad_workspace_bytes(rows, width, n, dy.dtype), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.adasum_embedding_grad(dy, ids, flat, 0, rows, workspace=work)
    torch.cuda.synchronize()
    assert torch.equal(flat, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adasum_embedding_grad(dy, ids, flat, 0, rows, workspace=work)
        looked = B.adasum_embedding(flat, 0, rows, width, ids)
    for rep in range(4):
        ids.copy_(make_ids(20 + rep, n, rows, ("few", "any", "one", "padded")[rep]).cuda())
        work.fill_(255)
        B.adasum_embedding_grad(dy, ids, eager, 0, rows)
        want = B.adasum_embedding(eager, 0, rows, width, ids)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(flat, eager) and torch.equal(looked, want), rep
    # the stream that a call names
    B.adasum_embedding_grad(dy, ids, flat.zero_(), 0, rows, stream=torch.cuda.current_stream())
    named = torch.empty_like(flat)
    side.wait_stream(torch.cuda.current_stream())
    B.adasum_embedding_grad(dy, ids, named, 0, rows, stream=side)
    side.synchronize()
    assert torch.equal(named, eager) and torch.equal(flat, eager)


def test_the_binding_refuses_wrong_shapes():
    flat, ids, dy = torch.zeros(80, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, 8, device="cuda")
    for bad in (lambda: B.adasum_embedding(flat, 1, 10, 8, ids), lambda: B.adasum_embedding(flat, 0, 10, 8, ids.float()),
                lambda: B.adasum_embedding(flat, 0, 10, 8, ids, out=dy[:3]), lambda: B.adasum_embedding(flat, 0, 10, 8, ids, out=dy.t()),
                lambda: B.adasum_embedding(flat, -1, 10, 8, ids), lambda: B.adasum_embedding_grad(dy[:3], ids, flat, 0, 10),
                lambda: B.adasum_embedding_grad(dy, ids, flat, 0, 11), lambda: B.adasum_embedding_grad(dy.t(), ids, flat, 0, 10),
                lambda: B.adasum_embedding_grad(dy, ids.cpu(), flat, 0, 10), lambda: B.adasum_embedding_grad(dy, ids, flat[::2], 0, 5)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.AdasumError) as e:
        B.adasum_embedding_grad(dy, ids, flat, 0, 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.ERR_WORKSPACE
