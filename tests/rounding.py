"""Running error analysis: a Num holds true values and a bound on how far a
float32 evaluation of the same expression may be off, in any order of its sums.
An operation rounds by at most half a step (U = 2^-24 relative), and the
hardware's approximations of 2^x, 1 / x are off by at most 2 U."""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # half a step, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}
FLUSH = 2.0 ** -126                  # results of the approximations below this may come out as 0


class Num:
    def __init__(self, v, e=None):
        self.v = np.asarray(v, np.float64)
        self.e = np.zeros_like(self.v) if e is None else e

    def _round(self, v, e, n=1):
        return Num(v, e + n * U * (np.abs(v) + e) + FLUSH)

    def __add__(self, o):
        o = o if isinstance(o, Num) else Num(o)
        return self._round(self.v + o.v, self.e + o.e)

    def __mul__(self, o):
        o = o if isinstance(o, Num) else Num(o)
        return self._round(self.v * o.v, np.abs(self.v) * o.e + self.e * np.abs(o.v) + self.e * o.e)

    def __getitem__(self, i):
        return Num(self.v[i], self.e[i])

    def sum(self, axis, slack=0):
        """A sum of n terms in any order has at most n roundings a term."""
        n = np.prod([self.v.shape[a] for a in np.atleast_1d(axis)]) + slack
        mag = (np.abs(self.v) + self.e).sum(axis=axis)
        return Num(self.v.sum(axis=axis), self.e.sum(axis=axis) + n * U * mag + FLUSH)

    def scaled(self, rel):
        """The same with a further relative error."""
        return Num(self.v, self.e + rel * (np.abs(self.v) + self.e))

    @staticmethod
    def where(on, a, b):
        return Num(np.where(on, a.v, b.v), np.where(on, a.e, b.e))


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1.0, e) / (1.0 + e)


def silu(z):
    """z / (1 + e^-z) and its derivative, z a Num.  The exponent's argument is
    rounded twice (2 |z| U relative in e), 2^x and the quotient add 2 U each,
    the sum and the product 1 each; where e overflows the value is below
    2^-120."""
    s = sigmoid(z.v)
    rel = (2 * np.abs(z.v) + 6) * U
    k = Num(s, s * rel + s * (1 - s) * z.e + FLUSH)
    val = Num(z.v * s, np.abs(z.v) * k.e + s * z.e + 2 * U * np.abs(z.v * s) + 2.0 ** -120)
    one_less = Num(1 - s, k.e + U)
    slope = k * (Num(np.ones_like(s)) + z * one_less)
    return val, Num(slope.v, slope.e + 2.0 ** -120)


def softplus(r):
    """log(1 + e^r) and its derivative: at most 12 roundings each, and the
    argument's error times the derivative (whose own derivative is below it)."""
    s = sigmoid(r.v)
    v = np.maximum(r.v, 0) + np.log1p(np.exp(-np.abs(r.v)))
    return Num(v, s * r.e + 12 * U * v + FLUSH), Num(s, s * r.e + 12 * U * s + FLUSH)


def exp_of(delta, A, more=0.0):
    """e^{delta A}: A log2 e and the product are rounded, 2^x is off by 2 U; a
    result below 2^-126 counts as 0.  more: further relative error of delta."""
    arg = delta.v * A
    rel = np.abs(arg) * (3 * U + more) + np.abs(A) * delta.e + 2 * U
    v = np.exp(arg)
    return Num(v, v * np.expm1(np.minimum(rel, 1.0)) + FLUSH)


def check(got, want, dtype, label):
    """got within want's bound and one rounding to its type."""
    got = np.asarray(got, np.float64)
    assert got.shape == want.v.shape, f"{label}: shape {got.shape} for {want.v.shape}"
    assert np.isfinite(got).all(), f"{label}: not finite"
    lim = want.e + HALF[dtype] * (np.abs(want.v) + want.e) + TINY[dtype]
    err = np.abs(got - want.v)
    bad = np.argwhere(err > lim)
    assert len(bad) == 0, f"{label}: {len(bad)} of {err.size} off, first {tuple(bad[0])}: {got[tuple(bad[0])]!r} for " \
                          f"{want.v[tuple(bad[0])]!r}, bound {lim[tuple(bad[0])]:.3g}"
