"""The operators between the layers as a training step uses them together, with those that fill a worker's buffer: a block of two linear
layers with an activation between them, norms, dropout, a gate and an fp32 residual stream; four workers, and the reduction."""
import numpy as np
import pytest
import torch

from between_util import in_8_bits, join, join_grad, kept
from layer_grads_util import f64, half_step
from oracle import adasum_oracle as O
from paper_2006_02924_amd import binding as B, workloads as W
from test_gpu_join import near
from test_gpu_linear_products import bound, near as near_product

pytestmark = pytest.mark.gpu

TOKENS, WIDTH, WIDE, K = 300, 192, 520, 4
NAMES = ["norm_weight", "norm_bias", "widen", "widen_bias", "narrow", "narrow_bias", "after_weight", "after_bias", "gate", "last_weight", "last_bias"]
SIZES = [WIDTH, WIDTH, WIDE * WIDTH, WIDE, WIDTH * WIDE, WIDTH, WIDTH, WIDTH, WIDTH, WIDTH, WIDTH]
OFFS = W.offsets_from_sizes(SIZES)
AT = dict(zip(NAMES, OFFS))
FIRST = dict(dropout=0.1, before_weight=AT["norm_weight"], before_bias=AT["norm_bias"])
SECOND = dict(dropout=0.2, after=True, residual_scale=0.75, after_weight=AT["after_weight"], after_bias=AT["after_bias"], gate=AT["gate"],
              before_weight=AT["last_weight"], before_bias=AT["last_bias"])


def parameters(dtype):
    g = torch.Generator().manual_seed(1)
    flat = torch.randn(OFFS[-1], generator=g) * 0.1
    for name in ("norm_weight", "after_weight", "last_weight"):
        flat[AT[name]:AT[name] + WIDTH] += 1.0
    flat[AT["widen"]:AT["widen"] + WIDE * WIDTH] *= 0.7
    return flat.to(dtype).cuda()


class Block:
    """What a program makes once: forms, weights in 8 bits, a workspace for everything."""

    def __init__(self, dtype, seed):
        self.first = B.Join(WIDTH, dtype, stream_dtype=torch.float32, seed=seed, **FIRST)
        self.second = B.Join(WIDTH, dtype, stream_dtype=torch.float32, seed=seed + 1, **SECOND)
        self.widen, self.narrow = B.Weight8(WIDE, WIDTH), B.Weight8(WIDTH, WIDE)
        need = [B.adasum_join_grad_workspace_bytes(self.second, TOKENS), B.adasum_join_grad_workspace_bytes(self.first, TOKENS)]
        for a, b in ((WIDTH, WIDE), (WIDE, WIDTH)):
            need += [B.adasum_linear_workspace_bytes(TOKENS, a, b, dtype), B.adasum_checkpoint_weight_grad_workspace_bytes(TOKENS, a, b, dtype)]
        self.work = torch.empty(max(need), dtype=torch.uint8, device="cuda")

    def step(self, params, x, residual, weight, grad, count):
        """One worker's step for the loss sum(weight * y); fills its gradient buffer."""
        w = self.work
        B.adasum_linear_store(params, AT["widen"], WIDE, WIDTH, out=self.widen)
        B.adasum_linear_store(params, AT["narrow"], WIDTH, WIDE, out=self.narrow)
        h1, y1 = B.adasum_join(self.first, params, x, residual, step=count)
        kept_y = B.adasum_checkpoint_store(y1)
        u = B.adasum_linear(self.widen, y1, params=params, bias_offset=AT["widen_bias"], workspace=w)
        kept_u = B.adasum_checkpoint_store(u)
        a = torch.nn.functional.gelu(u.float()).to(u.dtype)
        kept_a = B.adasum_checkpoint_store(a)
        v = B.adasum_linear(self.narrow, a, params=params, bias_offset=AT["narrow_bias"], workspace=w)
        h2, y2 = B.adasum_join(self.second, params, v, h1, step=count)
        dv, dh1 = B.adasum_join_grad(self.second, params, grad, x=v, h=h2, dy=weight, step=count, workspace=w)
        B.adasum_checkpoint_weight_grad(kept_a, dv, grad, AT["narrow"], bias_offset=AT["narrow_bias"], workspace=w)
        da = B.adasum_linear_grad(self.narrow, dv, workspace=w)
        du = B.adasum_checkpoint_act_grad(kept_u, da, "gelu")
        B.adasum_checkpoint_weight_grad(kept_y, du, grad, AT["widen"], bias_offset=AT["widen_bias"], workspace=w)
        dy1 = B.adasum_linear_grad(self.widen, du, workspace=w)
        dx, dres = B.adasum_join_grad(self.first, params, grad, h=h1, dy=dy1, dh=dh1, step=count, workspace=w)
        return dict(h1=h1, y1=y1, u=u, a=a, v=v, h2=h2, y2=y2, dv=dv, dh1=dh1, da=da, du=du, dy1=dy1, dx=dx, dres=dres, kept_y=kept_y, kept_a=kept_a)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_of_four_workers(dtype):
    params = parameters(dtype)
    flat = f64(params)
    g = torch.Generator().manual_seed(2)
    count = torch.tensor([3], dtype=torch.int64, device="cuda")
    grads = []
    for k in range(K):
        block = Block(dtype, 100 + 2 * k)
        x = torch.randn(TOKENS, WIDTH, generator=g).to(dtype).cuda()
        residual = torch.randn(TOKENS, WIDTH, generator=g).cuda()
        weight = (torch.randn(TOKENS, WIDTH, generator=g) * 0.05).to(dtype).cuda()
        grad = torch.full((OFFS[-1],), float("nan"), dtype=dtype, device="cuda")
        r = block.step(params, x, residual, weight, grad, count)
        n = {name: f64(t) for name, t in r.items() if isinstance(t, torch.Tensor)}
        masks = [kept(TOKENS, WIDTH, p, 100 + 2 * k + i, 3) for i, p in enumerate((0.1, 0.2))]
        # every operator from what it was given, by its definition
        h, y = join(FIRST, flat, f64(x), f64(residual), masks[0])
        near(r["h1"], h), near(r["y1"], y)
        h, y = join(SECOND, flat, n["v"], n["h1"], masks[1])
        near(r["h2"], h), near(r["y2"], y)
        w1, w2 = (in_8_bits(flat[AT[m]:AT[m] + WIDE * WIDTH].reshape(s), 128)[0] for m, s in (("widen", (WIDE, WIDTH)), ("narrow", (WIDTH, WIDE))))
        b1, b2 = flat[AT["widen_bias"]:][:WIDE], flat[AT["narrow_bias"]:][:WIDTH]
        for name, given, w, bias in (("u", "y1", w1, b1), ("v", "a", w2, b2), ("da", "dv", w2.T, 0.0), ("dy1", "du", w1.T, 0.0)):
            t8 = in_8_bits(n[given], 1)[0]
            near_product(r[name], t8 @ w.T + bias, bound(t8, w, w.shape[1], dtype))
        dv, dh1, sums = join_grad(SECOND, flat, n["v"], n["h2"], f64(weight), None, masks[1])
        near(r["dv"], dv), near(r["dh1"], dh1)
        for name, at in (("after_weight", "after_weight"), ("after_bias", "after_bias"), ("gate", "gate"), ("before_weight", "last_weight"),
                         ("before_bias", "last_bias")):
            near(grad[AT[at]:AT[at] + WIDTH], sums[name])
        dx, dres, sums = join_grad(FIRST, flat, None, n["h1"], n["dy1"], n["dh1"], masks[0])
        near(r["dx"], dx), near(r["dres"], dres)
        near(grad[AT["norm_weight"]:][:WIDTH], sums["before_weight"])
        near(grad[AT["norm_bias"]:][:WIDTH], sums["before_bias"])
        # the linear layers' from what was kept in 8 bits: a rounding to the type, and sums of 300 terms in fp32
        got = f64(grad)
        for layer, d, inputs in (("widen", n["du"], r["kept_y"]), ("narrow", n["dv"], r["kept_a"])):
            want = d.T @ f64(B.adasum_checkpoint_load(inputs))
            most = np.abs(d).T @ np.abs(f64(B.adasum_checkpoint_load(inputs)))
            at = slice(AT[layer], AT[layer] + want.size)
            assert (np.abs(got[at].reshape(want.shape) - want) <= half_step(dtype) * np.abs(want) + 300 * 2.0 ** -22 * most).all()
        assert grad.isfinite().all()
        grads.append(grad)
    out = B.adasum_reduce(grads, OFFS)
    err = O.rel_l2_per_layer(f64(out), O.adasum_reduce([f64(t) for t in grads], OFFS), OFFS)
    assert (err <= (1e-5 if dtype == torch.float32 else 2.0 ** -8)).all(), err      # a rounding to the type


def test_a_captured_step():
    """The step in one graph, replayed with new data and new masks, beside eager steps."""
    dtype = torch.bfloat16
    params, block, other = parameters(dtype), Block(dtype, 7), Block(dtype, 7)
    g = torch.Generator().manual_seed(3)
    x, weight = (torch.randn(TOKENS, WIDTH, generator=g).to(dtype).cuda() for _ in range(2))
    residual = torch.randn(TOKENS, WIDTH, generator=g).cuda()
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    grads = [torch.zeros(OFFS[-1], dtype=dtype, device="cuda") for _ in range(2)]
    other.step(params, x, residual, weight, grads[1], count)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.step(params, x, residual, weight, grads[0], count)
        count.add_(1)
    last = None
    for rep in range(4):
        x.copy_(torch.randn(TOKENS, WIDTH, generator=g))
        params.mul_(1.01)
        eager = other.step(params, x, residual, weight, grads[1], count)
        graph.replay()
        torch.cuda.synchronize()
        assert int(count) == rep + 1
        for name in ("y2", "h2", "dx", "dres", "du"):
            assert torch.equal(out[name], eager[name]), (rep, name)
        assert torch.equal(grads[0], grads[1]) and (last is None or not torch.equal(last, grads[0]))
        last = grads[0].clone()
