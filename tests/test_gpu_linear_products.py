"""Linear layers in 8-bit floating point against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from between_util import in_8_bits
from layer_grads_util import DTYPES, f64, half_step, least, within
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
KEPT = ["f32", "bf16", "f16"]


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def parts(weight):
    """(as it is, transposed, exponents) of a weight's bytes."""
    o, w = weight.outputs, weight.width
    ob, wb = -(-o // 128), -(-w // 128)
    data = weight.data.cpu()
    a, b = o * wb * 128, w * ob * 128
    number = lambda t: t.view(torch.float8_e4m3fn).double().numpy()
    panels = lambda t, rows: t.reshape(-1, rows, 64).transpose(1, 0, 2).reshape(rows, -1)
    return (panels(number(data[:a]), o), panels(number(data[a:a + b]), w),
            data[a + b:a + b + ob * wb].numpy().astype(np.int64).reshape(ob, wb) - 127)


def spread(seed, n, width, dtype):
    """Rows of many magnitudes, a row of zeros, and numbers of the smallest size."""
    x = rand(seed, n, width) * torch.exp2(torch.randint(-12 if dtype == torch.float16 else -40, 10, (n, 1), generator=torch.Generator().manual_seed(seed)).float())
    if n > 3:
        x[1] = 0.0
        x[2] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        x[3] = torch.finfo(dtype).max if dtype == torch.float16 else 1e30
    return x.to(dtype)


def bound(x, w, depth, out):
    """How far a sum of products of `depth` numbers may be from theirs: the matrix cores cut off rather than round in sums of 128 (a step
    of fp32 each), which are added up in turn; what is below fp32's range is lost.

    16-bit results come from the 8-bit cores, which align the eight products of consecutive channels to the largest power of two in them and
    keep 13 bits below it: seven of the eight lose less than 2^-13 of the largest each.  That is at most the product of the largest
    numbers that the eight channels have on either side."""
    def most(a):
        a = np.nan_to_num(np.abs(a), nan=0.0)
        return np.pad(a, ((0, 0), (0, -a.shape[1] % 8))).reshape(a.shape[0], -1, 8).max(2)
    off = (128 + depth / 128 + 16) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T) + (depth / 128 + 8) * 2.0 ** -126
    return off if out == torch.float32 else off + 7 * 2.0 ** -13 * (most(x) @ most(w).T)


def near(got, want, off):
    within(f64(got), want, np.where(np.isfinite(want), off + (half_step(got.dtype) + 2.0 ** -24) * (np.abs(want) + off) + least(got.dtype), 0.0))


@pytest.mark.parametrize("dtype", KEPT)
@pytest.mark.parametrize("outputs, width, lead", [(1, 1, 0), (3, 200, 1), (128, 128, 0), (130, 127, 5), (300, 1000, 8), (257, 384, 0)])
def test_weights_in_8_bits(dtype, outputs, width, lead):
    dtype = DTYPES[dtype]
    w = rand(outputs, outputs, width) * torch.exp2(rand(1, outputs, 1) * 3)
    if width > 2:
        w[0, 1], w[0, 2] = float("nan"), float("inf")
    if outputs > 128:
        w[128:, :128] = 0.0
    flat = torch.cat([rand(2, lead), w.reshape(-1), rand(3, 5)]).to(dtype)
    kept = B.adasum_linear_store(flat.cuda(), lead, outputs, width)
    values, exps = in_8_bits(f64(flat[lead:lead + w.numel()]).reshape(outputs, width), 128)
    q, turned, e = parts(kept)
    assert np.array_equal(e, exps)
    scale = np.ldexp(1.0, np.repeat(np.repeat(e, 128, 0), 128, 1))
    assert np.array_equal((q * scale[:outputs])[:, :width], values, equal_nan=True) and not q[:, width:].any()
    assert np.array_equal(turned[:, :outputs], q[:, :width].T, equal_nan=True) and not turned[:, outputs:].any()


SIZES = [(1, 1, 1), (1, 128, 128), (2, 7, 9), (16, 130, 64), (17, 300, 17), (33, 1000, 250), (100, 128, 300), (64, 4096, 128), (5, 24, 2000), (128, 512, 640),
         (257, 384, 256), (300, 1030, 520), (700, 256, 1024), (1, 8192, 100)]


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16"), ("f16", "bf16")], ids="-".join)
@pytest.mark.parametrize("n, width, outputs", SIZES)
def test_both_products(types, n, width, outputs):
    dtype, out = DTYPES[types[0]], DTYPES[types[1]]
    products(dtype, out, n, width, outputs, 0 if n % 2 else 3)


def products(dtype, out, n, width, outputs, gap):
    w = (rand(1, outputs, width) * 0.1).reshape(-1)
    bias = rand(2, outputs) * 2
    flat = torch.cat([rand(3, 3), w, bias]).to(torch.bfloat16).cuda()
    weight = B.adasum_linear_store(flat, 3, outputs, width)
    w8, _ = in_8_bits(f64(flat[3:3 + w.numel()]).reshape(outputs, width), 128)
    given = {"x": spread(4, n, width, dtype), "dy": spread(5, n, outputs, dtype)}
    if out == torch.float16:
        given = {k: t.clamp(-60, 60) for k, t in given.items()}
    for name, t in given.items():
        wide = torch.full((n, t.shape[1] + gap), float("nan"), dtype=dtype, device="cuda")
        wide[:, :t.shape[1]] = t.cuda()
        t8, _ = in_8_bits(f64(t), 1)
        there = outputs if name == "x" else width
        to = torch.full((n, there + gap), 3.0, dtype=out, device="cuda")
        rows = wide[:, :t.shape[1]]
        if name == "x":
            b = f64(bias.to(torch.bfloat16))
            B.adasum_linear(weight, rows, params=flat, bias_offset=3 + w.numel(), out=to[:, :there])
            near(to[:, :there], t8 @ w8.T + b, bound(t8, w8, width, out))
            near(B.adasum_linear(weight, rows, out_dtype=out), t8 @ w8.T, bound(t8, w8, width, out))
        else:
            B.adasum_linear_grad(weight, rows, out=to[:, :there])
            near(to[:, :there], t8 @ w8, bound(t8, w8.T, outputs, out))
        assert (to[:, there:] == 3.0).all()


def test_numbers_that_8_bits_hold_are_multiplied_exactly():
    """Small whole numbers: every product and sum is exact, in every order."""
    g = torch.Generator().manual_seed(1)
    for n, width, outputs in ((1, 640, 48), (130, 1000, 300), (520, 520, 512)):
        w = torch.randint(-8, 9, (outputs, width), generator=g).float()
        x, dy = torch.randint(-8, 9, (n, width), generator=g).float(), torch.randint(-8, 9, (n, outputs), generator=g).float()
        weight = B.adasum_linear_store(w.reshape(-1).cuda(), 0, outputs, width)
        assert torch.equal(B.adasum_linear(weight, x.cuda()).cpu().double(), x.double() @ w.double().t())
        assert torch.equal(B.adasum_linear_grad(weight, dy.cuda()).cpu().double(), dy.double() @ w.double())


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")], ids="-".join)
@pytest.mark.parametrize("n, width, outputs", [(3000, 300, 700), (2600, 1000, 520), (9000, 130, 260), (4100, 384, 1024), (8300, 300, 1030)])
def test_both_products_by_tiles(types, n, width, outputs):
    """As above, of sizes that do not go the way of few tokens."""
    dtype, out = DTYPES[types[0]], DTYPES[types[1]]
    assert B.adasum_linear_workspace_bytes(n, width, outputs, out) > 0
    products(dtype, out, n, width, outputs, 3)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n, width, outputs", [(12345, 100, 1100), (16640, 128, 1024), (9000, 384, 2050), (33000, 250, 520), (2300, 130, 515), (4100, 1000, 640),
                                              (70000, 64, 256), (257, 64, 60000), (8300, 300, 1030), (8300, 1030, 300)])
def test_many_tiles(n, width, outputs, out):
    """More tiles than workgroups, whole ones and others, few and many steps: whole numbers whose sums all types hold."""
    g = torch.Generator(device="cuda").manual_seed(1)
    small = lambda *shape: torch.randint(-1, 2, shape, generator=g, device="cuda").float() * (torch.rand(*shape, generator=g, device="cuda") < 0.4)
    w, bias = small(outputs, width), small(outputs)
    flat = torch.cat([w.reshape(-1), bias])
    weight = B.adasum_linear_store(flat, 0, outputs, width)
    for rep in range(2):
        x = small(n, width).bfloat16()
        want = x.float() @ w.t() + bias
        assert want.abs().max() <= 256
        assert torch.equal(B.adasum_linear(weight, x, params=flat, bias_offset=outputs * width, out_dtype=out).float(), want)
        dy = small(n, outputs).bfloat16()
        want = dy.float() @ w
        if out == torch.float32 or want.abs().max() <= 256:
            assert torch.equal(B.adasum_linear_grad(weight, dy, out_dtype=out).float(), want)
        else:
            assert torch.equal(B.adasum_linear_grad(weight, dy, out_dtype=out), want.to(out))


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [20, 20000])
def test_rows_that_are_no_numbers_stay_alone(n, out):
    width, outputs = 300, 140
    weight = B.adasum_linear_store((rand(1, outputs * width)).cuda(), 0, outputs, width)
    x = rand(2, n, width)
    clean = B.adasum_linear(weight, x.cuda(), out_dtype=out)
    x[3, 5], x[7, 299], x[n - 1, 130] = float("nan"), float("inf"), float("-inf")
    got = B.adasum_linear(weight, x.cuda(), out_dtype=out)
    bad = [3, 7, n - 1]
    rest = [i for i in range(n) if i not in bad]
    assert got[bad].isnan().all() and torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_magnitudes_at_the_ends(out):
    """Exponents of both ends of the range, apart and against each other."""
    width, outputs = 256, 1024
    for wide, small in ((1e30, 1e-30), (1e-36, 1.0), (1.0, 1e-38), (2.0 ** 127, 2.0 ** -100)):
        for n in (4, 4000):
            w, x = rand(1, outputs, width) * small, rand(2, n, width).clamp(-1.9, 1.9) * wide
            weight = B.adasum_linear_store(w.reshape(-1).cuda(), 0, outputs, width)
            w8, x8 = in_8_bits(f64(w), 128)[0], in_8_bits(f64(x), 1)[0]
            near(B.adasum_linear(weight, x.cuda(), out_dtype=out), x8 @ w8.T, bound(x8, w8, width, out))


def test_more_dimensions_no_rows_and_no_depth():
    weight = B.adasum_linear_store(rand(1, 40 * 24).cuda(), 0, 40, 24)
    x = rand(2, 3, 5, 24).cuda()
    assert torch.equal(B.adasum_linear(weight, x).view(15, 40), B.adasum_linear(weight, x.view(15, 24)))
    assert B.adasum_linear_grad(weight, torch.zeros(2, 0, 40, device="cuda")).shape == (2, 0, 24)
    empty = B.adasum_linear_store(torch.zeros(40, device="cuda"), 0, 40, 0)
    bias = rand(3, 40).cuda()
    assert torch.equal(B.adasum_linear(empty, torch.zeros(7, 0, device="cuda"), params=bias, bias_offset=0, out=torch.empty(7, 40, device="cuda")),
                       bias.expand(7, 40))


def test_rows_beyond_32_bits():
    n, width, outputs = (1 << 20) + 3, 2080, 16
    x = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    x[n - 1], x[0] = torch.linspace(-3, 3, width, device="cuda"), 1.0
    flat = rand(1, outputs * width).cuda()
    weight = B.adasum_linear_store(flat, 0, outputs, width)
    w8, _ = in_8_bits(f64(flat).reshape(outputs, width), 128)
    y = B.adasum_linear(weight, x)
    for row in (0, n - 1):
        x8, _ = in_8_bits(f64(x[row:row + 1]), 1)
        near(y[row:row + 1], x8 @ w8.T, bound(x8, w8, width, torch.bfloat16))
    assert int(torch.count_nonzero(y[1:n - 1])) == 0
    del x
    back = B.adasum_linear_grad(weight, y)
    y8, _ = in_8_bits(f64(y[n - 1:]), 1)
    near(back[n - 1:], y8 @ w8, bound(y8, w8.T, outputs, torch.bfloat16))
    assert int(torch.count_nonzero(back[1:n - 1])) == 0


@pytest.mark.parametrize("n", [3, 5000])
def test_captured_on_another_stream_and_with_a_workspace(n):
    width, outputs = 768, 520
    flat = rand(1, outputs * width + outputs).cuda()
    weight = B.Weight8(outputs, width)
    x, dy = rand(2, n, width).bfloat16().cuda(), rand(3, n, outputs).bfloat16().cuda()
    need = B.adasum_linear_workspace_bytes(n, width, outputs, torch.bfloat16)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    y, dx = torch.empty(n, outputs, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)

    def step(y, dx, work, **kw):
        B.adasum_linear_store(flat, 0, outputs, width, out=weight, **kw)
        y = B.adasum_linear(weight, x, params=flat, bias_offset=outputs * width, out=y, workspace=work, **kw)
        return y, B.adasum_linear_grad(weight, dy, out=dx, workspace=work, **kw)

    want = step(None, None, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(None, None, None, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y, dx, work)
    for rep in range(4):
        x.copy_(rand(10 + rep, n, width))
        flat.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        want = step(None, None, None)
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]), rep


def test_the_binding_refuses():
    flat, x = torch.zeros(4000, device="cuda"), torch.zeros(4, 40, device="cuda")
    weight = B.adasum_linear_store(flat, 0, 16, 40)
    for bad in (lambda: B.adasum_linear_store(flat, 0, 16, 40, out=B.Weight8(16, 41)), lambda: B.adasum_linear_store(flat, 3990, 16, 40),
                lambda: B.adasum_linear(weight, x[:, :39]), lambda: B.adasum_linear(weight, x, out=x), lambda: B.adasum_linear(weight, x.cpu()),
                lambda: B.adasum_linear(weight, x, params=flat, bias_offset=3990), lambda: B.adasum_linear_grad(weight, x),
                lambda: B.adasum_linear(weight, x, out_dtype=torch.float16, out=torch.zeros(4, 16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
