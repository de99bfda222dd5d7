"""Values in 64 bits with what the tensor-core products may be off by (before an output's own rounding), carried through
the formulas.

A product's sum of n terms: the terms are exact in fp32 (8-bit mantissas), every addition is good to one unit, 2^-23 (the tensor
cores cut), and there are no more than n + 8 of them.  The exponential is good to 2 + 1.173 |x| units and the fast division to 2
(CUDA's stated bounds), so a sigmoid s of x to s ((1 - s) (2 + 1.173 |x|) + 4) units.  An operand rounded to bf16 is off by
2^-8 of its value at most.
"""
import torch

UNIT = 2.0 ** -23
BF16_HALF = 2.0 ** -8


def dot(a, ea, b, eb):
    """a @ b^T of a (off by ea) and b (off by eb; None = exact)."""
    v = a @ b.T
    size = (a.abs() + (0 if ea is None else ea)) @ (b.abs() + (0 if eb is None else eb)).T
    e = (a.shape[1] + 8) * UNIT * size
    if ea is not None:
        e = e + ea @ b.abs().T
    if eb is not None:
        e = e + (a.abs() + (0 if ea is None else ea)) @ eb.T
    return v, e


def sigmoid(x, ex):
    s = torch.sigmoid(x)
    return s, s * (1 - s) * ex + 0.05 * ex * ex + s * ((1 - s) * (2 + 1.173 * (x.abs() + ex)) + 4) * UNIT + 1e-37


def times(a, ea, b, eb):
    v = a * b
    e = a.abs() * eb + b.abs() * ea + ea * eb
    return v, e + UNIT * (v.abs() + e)


def plus(a, ea, b, eb):
    v, e = a + b, ea + eb
    return v, e + UNIT * (v.abs() + e)


def to_bf16(v, e):
    return v, e + BF16_HALF * (v.abs() + e) + 1e-38


def silu(x, ex):
    return times(x, ex, *sigmoid(x, ex))


def silu_grad(x, ex):
    """s (1 + x (1 - s))"""
    s, es = sigmoid(x, ex)
    r, er = plus(torch.ones_like(s), torch.zeros_like(s), -s, es)
    return times(s, es, *plus(torch.ones_like(s), torch.zeros_like(s), *times(x, ex, r, er)))


def gelu(x, ex):
    """0.5 x (1 + erf(x / sqrt 2)): erff is good to 2 units of its value, its argument to one; |gelu'| < 1.13."""
    v = torch.nn.functional.gelu(x)
    return v, 1.13 * ex + 0.5 * x.abs() * 6 * UNIT + 2 * UNIT * v.abs()


def gelu_grad(x, ex):
    """Phi(x) + x phi(x), in absolute terms: |gelu''| < 0.8; Phi to 4 units, the exponential to 2 + 1.173 x^2 / 2."""
    c = 0.5 * (1 + torch.erf(x * 0.5 ** 0.5))
    d = x * torch.exp(-0.5 * x * x) * 0.3989422804014327
    return c + d, 0.8 * ex + 4 * UNIT + (8 + 0.6 * x * x) * UNIT * d.abs()


def act(kind, x, ex):
    return (x, ex) if kind == 0 else silu(x, ex) if kind == 1 else gelu(x, ex)


def act_grad(kind, x, ex):
    return silu_grad(x, ex) if kind == 1 else gelu_grad(x, ex)


def check(got, v, e, what=""):
    """got, rounded once to its type, lies within the bound everywhere."""
    half = torch.finfo(got.dtype).eps / 2
    bound = e + half * (v.abs() + e) + torch.finfo(got.dtype).tiny
    diff = (got.double() - v).abs()
    bad = ~(diff <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {(diff / bound).max().item():.3g} times it"


def ffn(x, wgu, wd):
    """One expert's rows in 64 bits: out, its bound, and what the gradients need."""
    f = wd.shape[1]
    z, ez = dot(x, None, wgu, None)
    g, eg, u, eu = z[:, :f], ez[:, :f], z[:, f:], ez[:, f:]
    h, eh = to_bf16(*times(*silu(g, eg), u, eu))
    return dot(h, eh, wd, None), (g, eg, u, eu, h, eh)


def ffn_grads(x, wgu, wd, dy):
    """dx, dw_gate_up, dw_down of one expert, each with its bound (the summed-over rows count as terms)."""
    _, (g, eg, u, eu, h, eh) = ffn(x, wgu, wd)
    dh, edh = dot(dy, None, wd.T, None)
    du, edu = to_bf16(*times(dh, edh, *silu(g, eg)))
    dg, edg = to_bf16(*times(*times(dh, edh, u, eu), *silu_grad(g, eg)))
    d, ed = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    return dot(d, ed, wgu.T, None), dot(d.T, ed.T, x.T, None), dot(dy.T, None, h.T, eh.T)
