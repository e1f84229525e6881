"""Weight gradients whose sums are exact in fp32: whole numbers, of which every token's products count in every element, and fp32 numbers
that all three bf16 parts are needed for.  What is stored then has one value only, whatever the order of the sums."""
import torch

from layer_grads_util import DTYPES

CODES = {"f32": 0, "bf16": 1, "f16": 2}

# dtype, out, tokens, outputs, width, edge of a workgroup's square, parts that are joined
CASES = [
    # squares of 256 without parts: one step, whole steps only, and steps with a rest; outputs and channels that are multiples of eight
    # and of the square, or neither; every type of result
    ("bf16", "bf16", 300, 4096, 4096, 256, 1), ("bf16", "f32", 256, 4096, 4000, 256, 1), ("bf16", "f16", 100, 8192, 4096, 256, 1),
    ("f16", "f16", 300, 4096, 4096, 256, 1), ("f16", "f32", 321, 4096, 4097, 256, 1), ("f16", "bf16", 640, 4104, 4000, 256, 1),
    ("f32", "f32", 300, 4096, 4096, 256, 1), ("f32", "bf16", 128, 4104, 4000, 256, 1), ("f32", "f16", 500, 4096, 4095, 256, 1),
    ("bf16", "f32", 300, 4093, 4096, 256, 1), ("f16", "f16", 200, 4091, 4092, 256, 1), ("f32", "f32", 200, 4101, 4094, 256, 1),
    # with parts, the last of which may be shorter
    ("bf16", "bf16", 16400, 1024, 1000, 256, 16), ("bf16", "f32", 16384, 4096, 1024, 256, 4), ("bf16", "f32", 16400, 1021, 1000, 256, 16),
    ("f16", "f16", 16399, 1024, 1024, 256, 16), ("f16", "f32", 16400, 1023, 1000, 256, 16),
    ("f32", "f32", 4093, 1024, 4096, 256, 4), ("f32", "bf16", 9000, 1024, 1024, 256, 16), ("f32", "f32", 9000, 1021, 1024, 256, 16),
    # squares of 128, without and with parts
    ("bf16", "bf16", 777, 1024, 1024, 128, 1), ("f16", "f32", 256, 1000, 2048, 128, 1), ("f32", "f32", 300, 1024, 1021, 128, 1),
    ("bf16", "f32", 40000, 70, 40, 128, 157), ("f16", "f16", 8192, 64, 64, 128, 64), ("f32", "bf16", 40000, 70, 40, 128, 250),
    ("bf16", "bf16", 2048, 5, 1024, 128, 32), ("f16", "f16", 500, 7, 130, 128, 8), ("f16", "bf16", 5000, 1, 130, 128, 40),
    ("f32", "f32", 8192, 7, 33, 128, 128),
]


def whole_numbers(n, outputs, width, seed, device):
    """dy and x without zeros: dy up to 7, x up to 3 in magnitude, sums of at most 21 n."""
    g = torch.Generator(device=device).manual_seed(seed)

    def some(most, *shape):
        v = torch.randint(1, most + 1, shape, generator=g, device=device)
        return torch.where(torch.rand(shape, generator=g, device=device) < 0.5, -v, v).float()

    assert 21 * n < 1 << 24
    return some(7, n, outputs), some(3, n, width)


def three_parts(n, outputs, width, seed, device):
    """dy of fp32: some 1 + 2^-9 + 2^-17 of either sign, at most 40 of a column (zeros otherwise); x up to 3: sums below 128, in units of
    2^-17.  Every token has one where there are as many outputs as tokens between two of a column."""
    dy, x = whole_numbers(n, outputs, width, seed, device)
    apart = -(-n // 40)
    there = (torch.arange(n, device=device)[:, None] + 7 * torch.arange(outputs, device=device)) % apart == 0
    dy = dy.sign() * (1 + torch.where(dy.abs() > 3, 2.0 ** -9, -2.0 ** -9) + torch.where(dy.abs() % 2 == 1, 2.0 ** -17, -2.0 ** -17))
    return torch.where(there, dy, torch.zeros_like(dy)), x


def inputs(case, kind, device, seed=1):
    """dy and x in the case's type, which holds them exactly."""
    dtype, _, n, outputs, width = case[:5]
    dy, x = (three_parts if kind == "three parts" else whole_numbers)(n, outputs, width, seed, device)
    t = DTYPES[dtype]
    assert torch.equal(dy.to(t).float(), dy) and torch.equal(x.to(t).float(), x)
    return dy.to(t), x.to(t)


def gradients(dy, x, old_weight, old_bias, out):
    """Weight's and bias's gradient: sums that fp64 and fp32 hold exactly, rounded once.  (fp32 holds them, so a result of 16 bits comes
    from fp32 without a rounding before.)"""
    d = dy.double()
    weight = torch.matmul(d.t().contiguous(), x.double()) + old_weight.double()
    bias = d.sum(0) + old_bias.double()
    for v in (weight, bias):
        assert torch.equal(v.float().double(), v)
    return weight.float().to(out), bias.float().to(out)
