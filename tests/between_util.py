"""What the tests of the operators between the layers compare with: definitions in 64 bits, and how far fp32 may be from them.

The bounds are running error analyses: beside every array its error, by the rules for one rounding (U32 of the result) and for sums
(a sum of n terms in a tree over lanes that add up to 16 terms each: at most DEPTH roundings on the way of any term)."""
import numpy as np

from layer_grads_util import U32

DEPTH = 40      # 16 terms of a lane, 6 steps over a wave, 16 waves of a workgroup, and the division
PHILOX = (0xD2511F53, 0xCD9E8D57)
WEYL = (0x9E3779B9, 0xBB67AE85)


def philox(counter, key):
    """Philox4x32-10 of arrays of 32-bit words."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = list(key)
    for _ in range(10):
        a, b = c[0] * np.uint64(PHILOX[0]), c[2] * np.uint64(PHILOX[1])
        low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> shift) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[i] + WEYL[i]) % 2 ** 32 for i in range(2)]
    return c


def numbers(n, width, seed, step):
    """u(t, j) of adasum_dropout."""
    granules = -(-width // 8)
    t, g = np.meshgrid(np.arange(n), np.arange(granules), indexing="ij")
    seed, step = seed % 2 ** 64, step % 2 ** 64
    words = philox([g, t, np.full(g.shape, step % 2 ** 32), np.full(g.shape, step >> 32)], [seed % 2 ** 32, seed >> 32])
    halves = [h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return np.stack(halves, axis=2).reshape(n, granules * 8)[:, :width]


def kept(n, width, p, seed, step=0):
    """The mask, and the factor of what is kept."""
    limit = int(np.floor(65536 * p + 0.5))
    return numbers(n, width, seed, step) >= limit, 0.0 if limit == 65536 else 65536 / (65536 - limit)


class Bounded:
    """A value in 64 bits and how far the computed one may be from it."""

    def __init__(self, v, e=0.0):
        self.v = np.asarray(v, dtype=np.float64)
        self.e = np.broadcast_to(np.asarray(e, dtype=np.float64), self.v.shape)

    def _of(self, v, e):
        return Bounded(v, e + U32 * (np.abs(v) + e) + 2.0 ** -149)

    def __add__(self, o):
        return self._of(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        return self._of(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        return self._of(self.v * o.v, self.e * np.abs(o.v) + np.abs(self.v) * o.e + self.e * o.e)

    def mean(self):
        """Over a row."""
        n = self.v.shape[1]
        e = self.e.sum(1, keepdims=True) / n
        return Bounded(self.v.mean(1, keepdims=True), e + DEPTH * U32 * (np.abs(self.v).mean(1, keepdims=True) + e))

    def column_sums(self, depth):
        e = self.e.sum(0)
        return Bounded(self.v.sum(0), e + depth * U32 * (np.abs(self.v).sum(0) + e))


def const(v):
    """A number that fp32 may have to round."""
    return Bounded(v, U32 * np.abs(np.asarray(v, dtype=np.float64)))


def one_over_root(s):
    """1 / sqrt(s), two correctly rounded steps (s.e / s small or the bound is what the interval gives)."""
    v = 1 / np.sqrt(s.v)
    least = np.maximum(s.v - s.e, 1e-300)
    return Bounded(v, (1 / np.sqrt(least) - v) + 4 * U32 / np.sqrt(least))


def normed(t, norm, eps):
    """(hat, one over the spread) of rows."""
    if norm == "layer":
        t = t - t.mean()
    r = one_over_root((t * t).mean() + const(eps))
    return t * r, r


def norm_grad(d, w, hat, r, norm):
    a = d * w if w is not None else d
    back = a - hat * (a * hat).mean()
    if norm == "layer":
        back = back - a.mean()
        back = Bounded(back.v, back.e + 2 * U32 * (np.abs(a.v) + np.abs(hat.v * (a.v * hat.v).mean(1, keepdims=True))))   # another order of the three
    return r * back


def vector(flat, offset, width):
    """A vector of parameters as it is stored, or None."""
    return None if offset is None else Bounded(flat[offset:offset + width])


def join(form, flat, x, residual, keep=None):
    """(h, y) as Bounded; form: a dict of Join's arguments; keep: (mask, factor)."""
    width = x.shape[1]
    w = {name: vector(flat, form.get(name), width) for name in ("after_weight", "after_bias", "gate", "before_weight", "before_bias")}
    norm, eps = form.get("norm", "layer"), form.get("eps", 1e-5)

    def affine(t, side):
        t, _ = normed(t, norm, eps)
        t = t * w[side + "_weight"] if w[side + "_weight"] is not None else t
        return t + w[side + "_bias"] if w[side + "_bias"] is not None else t

    v = Bounded(x)
    if form.get("after"):
        v = affine(v, "after")
    if keep is not None:
        v = dropped(v, keep)
    if w["gate"] is not None:
        v = v * w["gate"]
    if residual is not None:
        v = const(form.get("residual_scale", 1.0)) * Bounded(residual) + v
    return v, affine(v, "before") if form.get("before", True) else None


def dropped(v, keep):
    mask, factor = keep
    with np.errstate(invalid="ignore"):
        out = v * const(factor)
    return Bounded(np.where(mask, out.v, 0.0), np.where(mask, out.e, 0.0))


def join_grad(form, flat, x, h, dy, dh, keep=None):
    """dx, dresidual and the vectors' gradients as Bounded."""
    width = (dy if dy is not None else dh).shape[1]
    rows = (dy if dy is not None else dh).shape[0]
    w = {name: vector(flat, form.get(name), width) for name in ("after_weight", "after_bias", "gate", "before_weight", "before_bias")}
    norm, eps, sums = form.get("norm", "layer"), form.get("eps", 1e-5), {}
    depth = -(-rows // 256) + 32 + 8      # a lane's rows (at least one of 256 workgroups has it), those that a workgroup has at once, and the end
    d = None
    if form.get("before", True):
        hat, r = normed(Bounded(h), norm, eps)
        g = Bounded(dy)
        sums["before_weight"], sums["before_bias"] = (g * hat).column_sums(depth), g.column_sums(depth)
        d = norm_grad(g, w["before_weight"], hat, r, norm)
    if dh is not None:
        d = Bounded(dh) if d is None else d + Bounded(dh)
    dresidual = const(form.get("residual_scale", 1.0)) * d
    dv = dropped(d, keep) if keep is not None else d
    if form.get("after") or w["gate"] is not None:
        v = Bounded(x)
        if form.get("after"):
            hat, r = normed(v, norm, eps)
            v = hat * w["after_weight"] if w["after_weight"] is not None else hat
            v = v + w["after_bias"] if w["after_bias"] is not None else v
        # (what is dropped adds nothing, whatever it holds)
        with np.errstate(invalid="ignore"):
            t = dv * v
        if keep is not None:
            t = Bounded(np.where(keep[0], t.v, 0.0), np.where(keep[0], t.e, 0.0))
        sums["gate"] = t.column_sums(depth)
        if w["gate"] is not None:
            dv = dv * w["gate"]
        if form.get("after"):
            sums["after_weight"], sums["after_bias"] = (dv * hat).column_sums(depth), dv.column_sums(depth)
            dv = norm_grad(dv, w["after_weight"], hat, r, norm)
    return dv, dresidual, sums


# ---- 8-bit floating point ---------------------------------------------------------------

def e4m3(v):
    """The nearest e4m3 number of values of at most 448 (fp64), ties to even; NaN for what is not finite."""
    fine = np.isfinite(v)
    a = np.where(fine, v, 0.0)
    step = np.ldexp(1.0, np.maximum(np.frexp(a)[1] - 1, -6) - 3)
    return np.where(fine, np.rint(a / step) * step, np.nan)


def exponent(block):
    """The least e >= -120 with max |x| <= 448 * 2^e over the finite values."""
    most = np.abs(np.where(np.isfinite(block), block, 0.0)).max(initial=0.0)
    e = max(-120, int(np.frexp(most)[1]) - 12) if most else -120      # 448 * 2^e is below it
    while most > np.ldexp(448.0, e):
        e += 1
    return e


def in_8_bits(x, tall):
    """(values, exponents) of blocks of `tall` x 128."""
    n, width = x.shape
    out = np.zeros((n, width))
    exps = np.zeros((-(-n // tall), -(-width // 128)), dtype=np.int64)
    for i in range(exps.shape[0]):
        for j in range(exps.shape[1]):
            at = slice(i * tall, (i + 1) * tall), slice(j * 128, (j + 1) * 128)
            exps[i, j] = exponent(x[at])
            with np.errstate(invalid="ignore"):
                out[at] = e4m3(np.ldexp(x[at], -exps[i, j])) * np.ldexp(1.0, exps[i, j])
    return out, exps
