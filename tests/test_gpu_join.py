"""The join of a block with its residual stream, and its gradient, against their definitions in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from between_util import join, join_grad, kept
from layer_grads_util import DTYPES, f64, half_step, least, within
from paper_2006_02924_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")]
SHAPES = [(1, 1), (3, 7), (40, 16), (5, 33), (1, 128), (37, 129), (30, 512), (70, 1000), (600, 1024), (9, 1025), (5, 2047), (4, 4096), (3, 4097), (2, 8191), (5, 8192)]
SEED = 0xFEDCBA9876543210


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def strided(t, gap):
    wide = torch.full((t.shape[0], t.shape[1] + gap), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t.cuda()
    return wide[:, :t.shape[1]]


def offsets(width, named, lead=3):
    """Places of the vectors, with gaps between them."""
    return {name: lead + i * (width + 2) for i, name in enumerate(named)}


def parameters(seed, form, width, dtype):
    flat = rand(seed, 3 + 5 * (width + 2) + 7) * 0.3
    for name in ("after_weight", "gate", "before_weight"):
        if name in form:
            flat[form[name]:form[name] + width] += 1.0
    return flat.to(dtype)


def near(got, want):
    """One rounding to the type behind the error of what is rounded.  A value from the type's largest and half a step on rounds to an
    infinity (fp16: 65520; rows without a spread have gradients of 1 / eps), so that is what must come of it; what is as near to
    that as its error may come out on either side."""
    dtype, v = got.dtype, want.v
    tol = want.e + half_step(dtype) * (np.abs(v) + want.e) + least(dtype)
    f = torch.finfo(dtype)
    limit = f.max + 2.0 ** np.floor(np.log2(f.max)) * f.eps / 2
    g = f64(got)
    beyond, either = np.abs(v) - want.e >= limit, np.isfinite(v) & (np.abs(np.abs(v) - limit) <= want.e)
    v = np.where(beyond, np.copysign(np.inf, v), v)
    v = np.where(either & np.isinf(g), g, v)
    within(g, v, np.where(np.isfinite(v), tol, 0.0))


ALL = ("after_weight", "after_bias", "gate", "before_weight", "before_bias")
FORMS = [
    dict(),                                                                        # norm alone
    dict(names=("before_weight", "before_bias"), dropout=0.1),                      # dropout, residual, norm
    dict(names=("before_weight",), norm="rms", eps=1e-6),
    dict(names=ALL, after=True, dropout=0.25, residual_scale=0.75),
    dict(names=("after_weight", "gate"), after=True, before=False, norm="rms", residual_scale=-1.25, dropout=0.1),
    dict(names=("gate",), before=False),
    dict(names=("gate", "before_bias"), dropout=0.5),
    dict(after=True, before=False),
]


def build(form, width, dtype, stream):
    form = dict(form)
    form.update(offsets(width, form.pop("names", ())))
    return form, B.Join(width, dtype, stream_dtype=stream, seed=SEED, **form)


def mask_of(form, n, width, step=0):
    p = form.get("dropout", 0.0)
    return kept(n, width, p, SEED, step) if p else None


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("k", range(len(FORMS)))
@pytest.mark.parametrize("n, width", SHAPES[::2])
def test_forward(types, k, n, width):
    forward(types, k, n, width, 0 if k % 2 else 3)


@pytest.mark.parametrize("k", [1, 3])
@pytest.mark.parametrize("n, width", SHAPES[1::2])
def test_forward_of_other_sizes(k, n, width):
    forward(("bf16", "bf16"), k, n, width, 8)


def forward(types, k, n, width, gap):
    dtype, stream = DTYPES[types[0]], DTYPES[types[1]]
    form, j = build(FORMS[k], width, dtype, stream)
    params = parameters(k, form, width, DTYPES[["f32", "bf16", "f16"][(k + n) % 3]])
    x, residual = rand(1, n, width).to(dtype), (rand(2, n, width) * 2 + 0.5).to(stream)
    if n > 2:
        x[1], residual[1] = 0.0, 0.0          # a row without spread
        x[2], residual[2] = 100.0, 0.25
    step = torch.tensor([11], dtype=torch.int64, device="cuda")
    want_h, want_y = join(form, f64(params), f64(x), f64(residual), mask_of(form, n, width, 11))
    h, y = strided(torch.zeros(n, width, dtype=stream), gap), strided(torch.zeros(n, width, dtype=dtype), gap) if j.before else None
    xs, rs = strided(x, gap), strided(residual, gap)
    B.adasum_join(j, params.cuda(), xs, rs, step=step, h=h, y=y)
    near(h, want_h)
    if j.before:
        near(y, want_y)
        assert gap == 0 or y._base[:, width:].isnan().all()
        # without h, the same y; with h in the stream's place, the same both
        assert torch.equal(B.adasum_join(j, params.cuda(), xs, rs, step=step, keep_h=False)[1], y)
    assert gap == 0 or h._base[:, width:].isnan().all()
    h2, y2 = B.adasum_join(j, params.cuda(), xs, rs, step=step, h=rs)
    assert h2 is rs and torch.equal(rs, h) and (y is None or torch.equal(y2, y))


@pytest.mark.parametrize("n, width", [(5, 96), (3, 1001)])
def test_without_a_stream(n, width):
    for k in (0, 3, 5):
        form, j = build(FORMS[k], width, torch.float32, None)
        params = parameters(k, form, width, torch.float32)
        x = rand(3, n, width)
        want_h, want_y = join(form, f64(params), f64(x), None, mask_of(form, n, width))
        h, y = B.adasum_join(j, params.cuda(), x.cuda())
        near(h, want_h)
        if j.before:
            near(y, want_y)


def backward_inputs(form, j, n, width, seed=5):
    dtype, stream = j.dtype, j.stream_dtype
    x = rand(seed, n, width).to(dtype) if j.reads_x else None
    h = (rand(seed + 1, n, width) * 2 + 0.5).to(stream) if j.before else None
    dy = rand(seed + 2, n, width).to(dtype) if j.before else None
    dh = rand(seed + 3, n, width).to(stream) if not j.before or form.get("dropout") else None
    if n > 2:
        for t in (x, h):
            if t is not None:
                t[1] = 0.0
    return x, h, dy, dh


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("k", range(len(FORMS)))
@pytest.mark.parametrize("n, width", SHAPES[::2])
def test_gradient(types, k, n, width):
    backward(types, k, n, width, 0 if k % 2 else 3)


@pytest.mark.parametrize("k", [1, 3])
@pytest.mark.parametrize("n, width", SHAPES[1::2] + [(2100, 48), (5000, 136), (1030, 1032)])
def test_gradient_of_other_sizes(k, n, width):
    backward(("bf16", "f32"), k, n, width, 8)


def backward(types, k, n, width, gap):
    dtype, stream = DTYPES[types[0]], DTYPES[types[1]]
    form, j = build(FORMS[k], width, dtype, stream)
    params = parameters(k, form, width, DTYPES[["f32", "bf16", "f16"][(k + n) % 3]])
    x, h, dy, dh = backward_inputs(form, j, n, width)
    grad_type = DTYPES[["bf16", "f32", "f16"][(k + width) % 3]]
    step = torch.tensor([4 + (9 << 33)], dtype=torch.int64, device="cuda")
    want_dx, want_dr, sums = join_grad(form, f64(params), *(None if t is None else f64(t) for t in (x, h, dy, dh)),
                                       mask_of(form, n, width, int(step)))
    dev = [None if t is None else strided(t, gap) for t in (x, h, dy, dh)]
    dx, dr = strided(torch.zeros(n, width, dtype=dtype), gap), strided(torch.zeros(n, width, dtype=stream), gap)
    start = (rand(9, params.numel()) * 0.1).to(grad_type)
    grad, more = start.cuda(), start.cuda()
    kw = dict(x=dev[0], h=dev[1], dy=dev[2], dh=dev[3], step=step)
    B.adasum_join_grad(j, params.cuda(), grad, dx=dx, dresidual=dr, **kw)
    B.adasum_join_grad(j, params.cuda(), more, accumulate=True, dresidual=False, **kw)
    near(dx, want_dx)
    near(dr, want_dr)
    for t in (dx, dr):
        assert gap == 0 or t._base[:, width:].isnan().all()
    touched = torch.zeros(params.numel(), dtype=torch.bool)
    for name in ALL:
        if name in form:
            at = slice(form[name], form[name] + width)
            touched[at] = True
            near(grad[at], sums[name])
            added = type(sums[name])(sums[name].v + f64(start[at]), sums[name].e + 2.0 ** -24 * (np.abs(sums[name].v) + sums[name].e + np.abs(f64(start[at]))))
            near(more[at], added)
    assert torch.equal(grad.cpu()[~touched], start[~touched]) and torch.equal(more.cpu()[~touched], start[~touched])
    if dev[3] is not None:      # the stream's gradient in the place of the one that came
        got = B.adasum_join_grad(j, params.cuda(), grad, dresidual=dev[3], **kw)
        assert got[1] is dev[3] and torch.equal(got[1], dr) and torch.equal(got[0], dx)


@pytest.mark.parametrize("k", [1, 3, 4])
@pytest.mark.parametrize("n, width", [(20000, 130), (7000, 600), (1700, 2050), (70000, 24), (2600, 1024), (700, 5000)])
def test_workgroups_that_go_round(k, n, width):
    """More rows than the workgroups have at once."""
    forward(("bf16", "f32"), k, n, width, 0)
    backward(("bf16", "bf16"), k, n, width, 0)


@pytest.mark.parametrize("k", range(len(FORMS)))
def test_gradient_against_differences(k):
    """The gradient of sum(y wy + h wh) along random directions, by the pass that fp64 makes of the definition."""
    n, width = 6, 40
    form, j = build(FORMS[k], width, torch.float32, None)
    params = parameters(k, form, width, torch.float32)
    x, residual = rand(1, n, width), rand(2, n, width)
    wy, wh = rand(3, n, width), rand(4, n, width)
    mask = mask_of(form, n, width)

    def loss(p, a, r):
        h, y = join(form, p, a, r, mask)
        return (h.v * f64(wh)).sum() + (0 if y is None else (y.v * f64(wy)).sum())

    h, _ = B.adasum_join(j, params.cuda(), x.cuda(), residual.cuda())
    grad = torch.zeros(params.numel(), device="cuda")
    dx, dr = B.adasum_join_grad(j, params.cuda(), grad, x=x.cuda() if j.reads_x else None, h=h if j.before else None,
                                dy=wy.cuda() if j.before else None, dh=wh.cuda())
    for seed, (i, got) in itertools.product((7, 8), enumerate((grad, dx, dr))):
        at = [f64(params), f64(x), f64(residual)]
        way, e = f64(rand(seed, *at[i].shape)), 2.0 ** -12
        more, less = [a.copy() for a in at], [a.copy() for a in at]
        more[i] += e * way
        less[i] -= e * way
        want = (loss(*more) - loss(*less)) / (2 * e)
        # e^2 / 6 of the third derivative along the way (rows of 40 with a spread near 1: below a thousand in all), and fp32's sums
        assert abs((f64(got) * way).sum() - want) <= e * e * 1e3 + 2.0 ** -17 * np.abs(f64(got) * way).sum()


def test_dropped_places_do_not_matter():
    """NaN and infinities of x in dropped places reach neither results nor gradients."""
    n, width = 20, 200
    form, j = build(dict(names=("gate", "before_weight"), dropout=0.5), width, torch.float32, None)
    params = parameters(1, form, width, torch.float32)
    mask = kept(n, width, 0.5, SEED)
    x, residual, dy = rand(1, n, width), rand(2, n, width), rand(3, n, width)
    dirty = torch.where(torch.from_numpy(mask[0]), x, torch.where(torch.arange(width) % 2 == 0, float("nan"), float("inf")))
    out = []
    for t in (x, dirty):
        h, y = B.adasum_join(j, params.cuda(), t.cuda(), residual.cuda())
        grad = torch.zeros(params.numel(), device="cuda")
        out.append([h, y, grad, *B.adasum_join_grad(j, params.cuda(), grad, x=t.cuda(), h=h, dy=dy.cuda())])
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*out))
    # everything dropped: the stream goes on alone, x and the gate get nothing
    form["dropout"] = 1.0
    j = B.Join(width, torch.float32, seed=SEED, **form)
    h, _ = B.adasum_join(j, params.cuda(), dirty.cuda(), residual.cuda())
    assert torch.equal(h.cpu(), residual)
    grad = torch.ones(params.numel(), device="cuda")
    dx, _ = B.adasum_join_grad(j, params.cuda(), grad, x=dirty.cuda(), h=h, dy=dy.cuda())
    assert (dx == 0).all() and (grad[form["gate"]:form["gate"] + width] == 0).all()


def test_rows_that_are_no_numbers_stay_alone():
    n, width = 9, 1000
    form, j = build(FORMS[3], width, torch.bfloat16, None)
    params = parameters(3, form, width, torch.float32).cuda()
    x, residual = rand(1, n, width).bfloat16().cuda(), rand(2, n, width).bfloat16().cuda()
    clean = B.adasum_join(j, params, x, residual)
    x[4, 17], residual[6, 3] = float("nan"), float("inf")
    got = B.adasum_join(j, params, x, residual)
    rest = [i for i in range(n) if i not in (4, 6)]
    for a, b in zip(clean, got):
        assert torch.equal(a[rest], b[rest])
    assert got[1][4].isnan().all() and got[1][6].isnan().all()


def test_large_means_keep_their_digits():
    """A spread far below the mean: the statistics do not cancel."""
    n, width = 8, 768
    x = (rand(1, n, width) + 4096.0)
    form, j = build(dict(), width, torch.float32, None)
    _, y = B.adasum_join(j, None, x.cuda())
    near(y, join(form, np.zeros(0), f64(x), None)[1])
    want = torch.nn.functional.layer_norm(x.double(), (width,), eps=1e-5)
    # values of 4096 have steps of 2^-12 / 4, the mean is off by a few of them at most
    assert (y.cpu().double() - want).abs().max() < 2.0 ** -10


def test_no_rows():
    form, j = build(FORMS[3], 40, torch.float32, None)
    params = parameters(3, form, 40, torch.float32).cuda()
    none = torch.zeros(0, 40, device="cuda")
    assert [t.shape for t in B.adasum_join(j, params, none, none)] == [(0, 40)] * 2
    grad = torch.full_like(params, 2.0)
    B.adasum_join_grad(j, params, grad, x=none, h=none, dy=none, dh=none, accumulate=True)
    assert (grad == 2.0).all()
    B.adasum_join_grad(j, params, grad, x=none, h=none, dy=none, dh=none)
    zero = torch.zeros_like(params, dtype=torch.bool)
    for name in ALL:
        zero[form[name]:form[name] + 40] = True
    assert (grad[zero] == 0).all() and (grad[~zero] == 2.0).all()


def test_rows_beyond_32_bits():
    n, width = (1 << 20) + 3, 2080
    j = B.Join(width, torch.bfloat16, before_weight=0, before_bias=width, norm="rms")
    params = torch.ones(2 * width, device="cuda")
    x = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    x[n - 1], x[0] = torch.linspace(-3, 3, width, device="cuda"), 2.0
    _, y = B.adasum_join(j, params, x, keep_h=False)
    want = x[n - 1].double() / (x[n - 1].double().square().mean() + 1e-5).sqrt() + 1
    assert (y[n - 1].double() - want).abs().max() < 2.0 ** -6 and (y[0] == 2.0).all() and (y[1:n - 1] == 1.0).all()
    grad = torch.zeros(2 * width, device="cuda")
    dx, _ = B.adasum_join_grad(j, params, grad, h=x, dy=x, dresidual=False)
    assert int(torch.count_nonzero(dx[1:n - 1])) == 0 and torch.equal(grad[width:], (x[0].float() + x[n - 1].float()))


def test_captured_on_another_stream_and_twice_at_once():
    n, width = 300, 768
    form, j = build(FORMS[3], width, torch.bfloat16, torch.float32)
    params = parameters(3, form, width, torch.float32).cuda()
    x, residual, dy = rand(1, n, width).bfloat16().cuda(), rand(2, n, width).cuda(), rand(3, n, width).bfloat16().cuda()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    grads = [torch.zeros_like(params) for _ in range(2)]
    work = [torch.empty(B.adasum_join_grad_workspace_bytes(j, n), dtype=torch.uint8, device="cuda") for _ in range(2)]
    dx, dr, h, y = torch.empty_like(x), torch.empty_like(residual), torch.empty_like(residual), torch.empty_like(x)

    def both(which, out, **kw):
        hh, yy = B.adasum_join(j, params, x, residual, step=step, h=out[0], y=out[1], **kw)
        return [hh, yy, *B.adasum_join_grad(j, params, grads[which], x=x, h=hh, dy=dy, dh=residual, step=step, dx=out[2], dresidual=out[3],
                                            workspace=work[which], **kw), grads[which]]

    want = [t.clone() for t in both(0, (None,) * 4)]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = [both(k, (None,) * 4, stream=s) for k, s in enumerate(sides)]
    torch.cuda.synchronize()
    for run in got:
        assert all(torch.equal(a, b) for a, b in zip(run, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(1, (h, y, dx, dr))
        step.add_(1)
    for rep in range(4):
        x.copy_(rand(20 + rep, n, width))
        graph.replay()
        torch.cuda.synchronize()
        step.sub_(1)
        eager = both(0, (None,) * 4)
        assert all(torch.equal(a, b) for a, b in zip(eager, (h, y, dx, dr, grads[1]))), rep
        step.add_(1)


def test_the_binding_refuses():
    x = torch.zeros(4, 40, device="cuda")
    j = B.Join(40, torch.float32, gate=0)
    flat = torch.zeros(40, device="cuda")
    for bad in (lambda: B.adasum_join(j, flat[:39], x), lambda: B.adasum_join(j, flat.cpu(), x), lambda: B.adasum_join(j, flat, x, x[:3]),
                lambda: B.adasum_join(j, flat, x.half()), lambda: B.adasum_join(j, flat, x, x.half()), lambda: B.adasum_join(j, flat, x.t()),
                lambda: B.adasum_join(j, flat, x, h=x.half()), lambda: B.adasum_join(j, flat, x, y=x[:3]),
                lambda: B.adasum_join(B.Join(40, torch.float32, before=False), flat, x, y=x.clone()),
                lambda: B.adasum_join_grad(j, flat, None, x=x, h=x, dy=x), lambda: B.adasum_join_grad(j, flat, flat, x=x[:3], h=x, dy=x),
                lambda: B.adasum_join_grad(j, flat, flat, x=x, h=x, dy=x, workspace=flat.cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.AdasumError):
        B.adasum_join(B.Join(8200, torch.float32), None, torch.zeros(1, 8200, device="cuda"))
    with pytest.raises(B.AdasumError):
        B.adasum_join(B.Join(40, torch.float32), None, x, y=x)
