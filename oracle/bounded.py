"""Float64 arrays that carry a bound of the error a float32 computation of the same expression may have.

``v`` is the value, ``e`` the bound in units of 2**-24 (half a step of float32 relative to a value).  The rules are those of a
running error analysis: a sum or product adds one rounding of its result to what its operands bring along; a sum over an axis
is one rounding of the sum of absolute values for each level of additions, at most ``levels`` of them; elementary functions
bring ``own`` roundings of their result and what the argument's error makes of it.
"""
import numpy as np

LOG2E = 1.4426950408889634


class Bounded:
    __array_priority__ = 100

    def __init__(self, v, e=None):
        self.v = np.asarray(v, np.float64)
        self.e = np.zeros_like(self.v) if e is None else np.asarray(e, np.float64)

    def __add__(self, o):
        o = lift(o)
        v = self.v + o.v
        return Bounded(v, self.e + o.e + np.abs(v))

    __radd__ = __add__

    def __neg__(self):
        return Bounded(-self.v, self.e)

    def __sub__(self, o):
        return self + -lift(o)

    def __rsub__(self, o):
        return lift(o) + -self

    def __mul__(self, o):
        o = lift(o)
        v = self.v * o.v
        return Bounded(v, self.e * np.abs(o.v) + np.abs(self.v) * o.e + np.abs(v))

    __rmul__ = __mul__

    def __getitem__(self, i):
        return Bounded(self.v[i], self.e[i])

    def reshape(self, *s):
        return Bounded(self.v.reshape(*s), self.e.reshape(*s))

    def sum(self, axis, levels=None):
        levels = self.v.shape[axis] if levels is None else levels
        return Bounded(self.v.sum(axis), self.e.sum(axis) + levels * np.abs(self.v).sum(axis))


def lift(x):
    return x if isinstance(x, Bounded) else Bounded(x)


def exp(x):
    """2**(x log2 e): the scaled argument has two roundings, the function's approximation four."""
    x = lift(x)
    v = np.exp(x.v)
    return Bounded(v, v * (x.e + 2 * np.abs(x.v) + 4))


def sigmoid(x):
    """1 / (1 + e^-x): the error of e^-x counts by its share, 1 - sigmoid, of the denominator."""
    x = lift(x)
    t = np.exp(-np.abs(x.v))
    v = np.where(x.v >= 0, 1 / (1 + t), t / (1 + t))
    return Bounded(v, v * ((1 - v) * (x.e + 2 * np.abs(x.v) + 4) + 4))


def softplus(x):
    """max(x, 0) + log1p(e^-|x|): the logarithm by a series of some ten operations."""
    x = lift(x)
    t = np.exp(-np.abs(x.v))
    small = np.log1p(t)
    v = np.maximum(x.v, 0) + small
    return Bounded(v, x.e / (1 + np.exp(-x.v)) + small * (2 * np.abs(x.v) + 20) + v)


def log(x):
    x = lift(x)
    v = np.log(x.v)
    return Bounded(v, x.e / np.abs(x.v) + 4 * np.abs(v) + 4)
