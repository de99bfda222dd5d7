"""Values with rigorous error bounds: what an fp32 evaluation of a formula may be off by.

A Bounded holds the formula's value in 64 bits and a bound on the difference of any fp32 evaluation from it: the
operands' bounds are carried through, and every operation adds one rounding (half a unit, 2^-24 relative; a fused
multiply-add rounds less often, never more).  A sum of n terms in any order adds at most n roundings of the sum of
the terms' magnitudes.  `within` adds the rounding of the output to its type.
"""
import torch

U = 2.0 ** -24


class Bounded:
    def __init__(self, v, e=None):
        self.v = v.double() if torch.is_tensor(v) else torch.tensor(float(v), dtype=torch.float64)
        self.e = torch.zeros_like(self.v) if e is None else e

    @staticmethod
    def of(x):
        return x if isinstance(x, Bounded) else Bounded(x)

    def _rounded(self, v, e):
        return Bounded(v, e + U * (v.abs() + e))

    def __add__(self, o):
        o = Bounded.of(o)
        return self._rounded(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        o = Bounded.of(o)
        return self._rounded(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        o = Bounded.of(o)
        return self._rounded(self.v * o.v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e)

    def sum(self, dim, keepdim=False):
        n = self.v.shape[dim]
        mag = (self.v.abs() + self.e).sum(dim, keepdim=keepdim)
        return Bounded(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + 1.01 * n * U * mag)

    def rsqrt(self):
        """rsqrtf is good to 2 units (4 halves); the derivative at the lower end bounds the operand's share."""
        low = (self.v - self.e).clamp(min=1e-300)
        v = self.v.rsqrt()
        e = 0.5 * low.pow(-1.5) * self.e
        return Bounded(v, e + 4 * U * (v + e))

    def silu(self):
        """v / (1 + exp(-v)): |silu'| < 1.1; exponential, sum and quotient are good to 8 halves together."""
        v = self.v * torch.sigmoid(self.v)
        e = 1.1 * self.e
        return Bounded(v, e + 8 * U * (v.abs() + e) + 1e-38)

    def within(self, got, what=""):
        """got, rounded once to its type, lies within the bound everywhere."""
        out = torch.finfo(got.dtype).eps / 2
        bound = self.e + out * (self.v.abs() + self.e) + torch.finfo(got.dtype).tiny
        diff = (got.double() - self.v).abs()
        bad = ~(diff <= bound)
        assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst "
                               f"{(diff / bound).max().item():.3g} times it")
