"""The operators as a training step uses them together: an embedding, two linear layers with an activation between them, four
workers whose gradients fill flat buffers, and the reduction of those."""
import numpy as np
import pytest
import torch

from layer_grads_util import f64, phi
from oracle import adasum_oracle as O
from paper_2006_02924_amd import binding as B, workloads as W

pytestmark = pytest.mark.gpu

ROWS, WIDTH, WIDE, TOKENS, K = 300, 64, 160, 500, 4
SIZES = [ROWS * WIDTH, WIDE * WIDTH, WIDE, WIDTH * WIDE, WIDTH]       # table, widening layer, its bias, narrowing layer, its bias


def forward_and_backward(params, ids, weight, grad, offs, stream=None):
    """One worker's step for the loss sum(weight * y): keeps activations in 8 bits, fills its gradient buffer."""
    table, w1, b1, w2, b2 = (params[a:b].float() for a, b in zip(offs, offs[1:]))
    x = B.adasum_embedding(params, offs[0], ROWS, WIDTH, ids, scale=8.0, stream=stream)
    kept_x = B.adasum_checkpoint_store(x)
    u = (torch.addmm(b1, x.float(), w1.view(WIDE, WIDTH).t().contiguous())).to(params.dtype)
    kept_u = B.adasum_checkpoint_store(u)
    h = torch.nn.functional.gelu(u.float()).to(params.dtype)
    kept_h = B.adasum_checkpoint_store(h)
    dy = weight
    B.adasum_checkpoint_weight_grad(kept_h, dy, grad, offs[3], bias_offset=offs[4])
    dh = (dy.float() @ w2.view(WIDTH, WIDE)).to(params.dtype)
    du = B.adasum_checkpoint_act_grad(kept_u, dh, "gelu", out=dh)
    B.adasum_checkpoint_weight_grad(kept_x, du, grad, offs[1], bias_offset=offs[2])
    dx = (du.float() @ w1.view(WIDE, WIDTH)).to(params.dtype)
    B.adasum_embedding_grad(dx, ids, grad, offs[0], ROWS, scale=8.0)
    return kept_x, kept_u, kept_h, dh.clone(), dx


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_of_four_workers(dtype):
    offs = W.offsets_from_sizes(SIZES)
    g = torch.Generator().manual_seed(3)
    params = (torch.randn(offs[-1], generator=g) * 0.1).to(dtype).cuda()
    grads, wants = [], []
    for k in range(K):
        ids = torch.randint(0, ROWS, (TOKENS,), generator=g)
        ids[-7:] = -1
        weight = (torch.randn(TOKENS, WIDTH, generator=g) * 0.05).to(dtype).cuda()
        grad = torch.full((offs[-1],), float("nan"), dtype=dtype, device="cuda")
        kept_x, kept_u, kept_h, du, dx = forward_and_backward(params, ids.cuda(), weight, grad, offs)
        grads.append(grad)
        # every layer's gradient from what the step kept and passed on, in 64 bits
        x, u, h = (f64(B.adasum_checkpoint_load(c)) for c in (kept_x, kept_u, kept_h))
        d, dun, dxn = f64(weight), f64(du), f64(dx)
        table = np.zeros((ROWS, WIDTH))
        there = (ids >= 0).numpy()
        np.add.at(table, ids.numpy()[there], dxn[there])
        want = np.concatenate([8 * table.ravel(), (dun.T @ x).ravel(), dun.sum(0), (d.T @ h).ravel(), d.sum(0)])
        wants.append(want)
        eps = torch.finfo(dtype).eps / 2
        got = f64(grad)
        for a, b in zip(offs, offs[1:]):
            scale = np.abs(want[a:b]).max()
            # a rounding of each element to the type, and sums of 500 terms in fp32
            assert np.abs(got[a:b] - want[a:b]).max() <= (eps + 500 * 2.0 ** -22) * scale
        # the activation's gradient against the derivative of the kept input, by way of the pass that made it: du = dh * slope(u)
        p, density = phi(u)
        dh = f64((weight.float() @ params[offs[3]:offs[4]].float().view(WIDTH, WIDE)).to(dtype))
        assert np.abs(dun - dh * (p + u * density)).max() <= (eps + 2.0 ** -18) * np.abs(dh).max() * 1.2
    out = B.adasum_reduce(grads, offs)
    want = O.adasum_reduce([f64(t) for t in grads], offs)
    err = O.rel_l2_per_layer(f64(out), want, offs)
    assert (err <= (1e-5 if dtype == torch.float32 else 2e-3)).all(), err


def test_a_captured_step():
    """The library's part of a backward pass in one graph with the reduction, replayed with new data."""
    offs = W.offsets_from_sizes(SIZES)
    g = torch.Generator().manual_seed(4)
    dtype = torch.bfloat16
    kept = [B.adasum_checkpoint_store((torch.randn(TOKENS, w, generator=g)).to(dtype).cuda()) for w in (WIDTH, WIDE, WIDE)]
    ids = torch.randint(0, ROWS, (TOKENS,), generator=g).cuda()
    dy, dh = (torch.randn(TOKENS, w, generator=g).to(dtype).cuda() for w in (WIDTH, WIDE))
    grads = [torch.zeros(offs[-1], dtype=dtype, device="cuda") for _ in range(2)]
    out, eager_out = torch.empty_like(grads[0]), torch.empty_like(grads[0])
    plan = B.Plan(2, offs, dtype)
    need = max(B.adasum_checkpoint_weight_grad_workspace_bytes(TOKENS, a, b, dtype) for a, b in ((WIDE, WIDTH), (WIDTH, WIDE)))
    work = torch.empty(max(need, B.adasum_embedding_grad_workspace_bytes(ROWS, WIDTH, TOKENS, dtype)), dtype=torch.uint8, device="cuda")

    def backward(to):
        for k, grad in enumerate(grads):
            B.adasum_checkpoint_weight_grad(kept[2], dy, grad, offs[3], bias_offset=offs[4], workspace=work)
            du = B.adasum_checkpoint_act_grad(kept[1], dh, ("gelu", "silu")[k])
            B.adasum_checkpoint_weight_grad(kept[0], du, grad, offs[1], bias_offset=offs[2], workspace=work)
            B.adasum_embedding_grad(dy, ids, grad, offs[0], ROWS, workspace=work)
        plan.execute(grads, to)

    backward(eager_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        backward(out)
    for rep in range(4):
        dy.copy_(torch.randn(TOKENS, WIDTH, generator=g))
        dh.copy_(torch.randn(TOKENS, WIDE, generator=g))
        ids.copy_(torch.randint(-1, ROWS, (TOKENS,), generator=g))
        backward(eager_out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out), rep
