"""What the tests of the operators that fill a worker's gradient buffer compare with: definitions in 64 bits, and how far a result
may be from them."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f64": torch.float64}
PAIRS = [(a, b) for a in ("f32", "bf16", "f16") for b in ("f32", "bf16", "f16")] + [("f64", "f64")]
U32 = 2.0 ** -24


def half_step(dtype):
    """A rounding to this type: at most this much of the value ..."""
    return torch.finfo(dtype).eps / 2


def least(dtype):
    """... and at most this much where the type's steps get no finer (half of its smallest number; with some room for fp32 in between)."""
    f = torch.finfo(dtype)
    return f.smallest_normal * f.eps / 2 + 2.0 ** -140


def lane_u(dtype):
    """Half a step of the type that sums are formed in."""
    return 2.0 ** -53 if dtype == torch.float64 else U32


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, tol):
    """got and want agree where want is finite, and are the same infinity or NaN elsewhere."""
    got, want, tol = np.asarray(got), np.asarray(want), np.broadcast_to(np.asarray(tol), np.shape(want))
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    off = np.abs(got[~odd] - want[~odd])
    bad = ~(off <= tol[~odd])
    if bad.any():
        k = np.argmax(off - tol[~odd])
        raise AssertionError(f"{bad.sum()} of {bad.size} beyond: {got[~odd][k]!r} for {want[~odd][k]!r}, {off[k]:.3e} > {tol[~odd][k]:.3e}")


def keep(x):
    """Whole numbers and exponents of a checkpoint of the rows of x, by its definition (x as fp64)."""
    n, width = x.shape
    blocks = -(-width // 32)
    q, e = np.zeros((n, blocks * 32), dtype=np.int64), np.full((n, blocks), -120, dtype=np.int64)
    for b in range(blocks):
        part = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(part).all(axis=1)
        most = np.where(bad, 0.0, np.abs(np.where(bad[:, None], 0.0, part)).max(axis=1))
        ex = np.where(most > 0, np.frexp(most)[1] - 7, -120).clip(-120, None)
        v = np.clip(np.rint(np.ldexp(np.where(bad[:, None], 0.0, part), -ex[:, None])), -127, 127)
        q[:, 32 * b:32 * b + part.shape[1]] = v.astype(np.int64)
        e[:, b] = np.where(bad, -128, ex)
    return q, e


def values(q, e, width):
    """What they stand for."""
    step = np.where(e == -128, np.nan, np.ldexp(1.0, np.where(e == -128, 0, e).astype(int)))
    return (q * np.repeat(step, 32, axis=1))[:, :width]


def split(data, n, width):
    """The two arrays of a checkpoint's bytes."""
    blocks = -(-width // 32)
    a = data.cpu().view(torch.int8).numpy().astype(np.int64)
    return a[:n * blocks * 32].reshape(n, blocks * 32), a[n * blocks * 32:].reshape(n, blocks)


def phi(x):
    """Phi(x) and the density (fp64)."""
    t = torch.from_numpy(x)
    return (torch.erfc(-t / math.sqrt(2)) / 2).numpy(), np.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def sigmoid(x):
    return torch.sigmoid(torch.from_numpy(np.ascontiguousarray(x))).numpy()


def slope(x, act):
    """Derivative of the activation, and how far fp32 may be from it.

    The formulas take a few roundings and functions of a few units in the last place each; what grows with x is the
    rounding of an exponential's argument, whose size is x^2 / 2, |x| or |z|, and erfc's, twice that.  Below that comes
    what underflows."""
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        if act == "relu":
            return np.where(np.isnan(x), x, (x > 0) * 1.0), np.zeros_like(x)
        if act == "gelu":
            p, d = phi(x)
            return p + x * d, U32 * (16 + 4 * np.minimum(x * x, 400)) * (p + np.abs(x) * d) + 1e-36
        if act == "silu":
            h, o = sigmoid(x), sigmoid(-x)
            ho = np.where(np.isnan(x), x, np.where(np.abs(x) > 700, 0.0, x * h * o))
            return h + ho, U32 * (16 + 4 * np.minimum(np.abs(x), 200)) * (h + np.abs(ho)) + 1e-36
        y = np.clip(x, -60, 60)
        c, k = math.sqrt(2 / math.pi), 0.044715
        z = 2 * c * (y + k * y ** 3)
        h, o = sigmoid(z), sigmoid(-z)
        rest = y * h * o * 2 * c * (1 + 3 * k * y * y)
        return h + rest, U32 * (16 + 8 * np.minimum(np.abs(z), 200)) * (h + np.abs(rest)) + 1e-36
