"""The norms with an output in 8 bits against their definition in 64 bits.

A code is right if it is the e4m3 number nearest to some value that fp32 arithmetic may have given: the definition's value,
off by its bound, rounded at either end.  A scale and a sum have their bounds alone.
"""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests.bounds import Bounded, U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _g(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _gauss(shape, seed, dtype, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=_g(seed), device=DEV) * scale + mean).to(dtype)


def _inv(v, h, eps):
    return ((v * v).sum(1, keepdim=True) * Bounded(1.0 / h) + Bounded(eps)).rsqrt()


def _check_codes(s, w, eps, normalise, codes, scale):
    """s: what is normed (with its bound).  The code's value is s w 448 / max |s w|; the reciprocal is good to 2 units, 2^-23."""
    h = s.v.shape[1]
    p = s if w is None else s * Bounded(w)
    m = p.v.abs().amax(1, keepdim=True)
    em = (p.e + U * p.v.abs()).amax(1, keepdim=True)
    low = torch.full_like(m, 2.0 ** -110)
    m = torch.maximum(m, low)
    val = p.v * 448 / m
    err = p.e * 448 / m + val.abs() * (em / m + 6 * 2.0 ** -23)
    ends = [(val + k * err).float().to(F8).float() for k in (-1.0, 1.0)]
    got = codes.float()
    # an end in fp32 and then in 8 bits may itself be rounded: a unit of fp32 is in the bound
    assert ((got >= ends[0]) & (got <= ends[1])).all(), ((got < ends[0]) | (got > ends[1])).sum().item()
    full = Bounded(m, em) * Bounded(1.0 / 448)
    if normalise:
        full = full * _inv(s, h, eps)
    full = Bounded(full.v, full.e + 2 * U * full.v)
    full.within(scale[:, None], "scale")


def _want_sum(x, y, w, gate, kind, a, b, normalise, eps):
    h = x.shape[1]
    Y = Bounded(y)
    if normalise:
        Y = Y * _inv(Y, h, eps)
        if w is not None:
            Y = Y * Bounded(w)
    if gate is not None:
        Y = Y * Bounded(gate[:, None] if kind == binding.GATE_TOKEN else gate)
    # the factors' order is the kernel's own: one rounding more for each
    Y = Y * Bounded(float(b))
    Y = Bounded(Y.v, Y.e + 3 * U * Y.v.abs())
    return Bounded(x) * Bounded(float(a)) + Y


SIZES = [(1, 1), (1, 7168), (3, 33), (7, 1024), (296, 64), (297, 1024), (300, 2048), (600, 1027), (700, 2056), (900, 7168), (310, 8192), (320, 9000),
         (400, 4100), (333, 16384)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,h", SIZES)
def test_norm(T, h, dtype):
    x = _gauss((T, h), T + h, dtype, 2.0)
    for w in (None, _gauss((h,), 1, F32, 0.2, 1.0), _gauss((h,), 1, BF16, 0.2, 1.0)):
        for normalise in (True, False):
            codes, scale = binding.norm_quant(x, w, 1e-6, normalise=normalise)
            _check_codes(Bounded(x), w, 1e-6, normalise, codes, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,h", SIZES)
@pytest.mark.parametrize("kind", [binding.GATE_NONE, binding.GATE_CHANNEL, binding.GATE_TOKEN, binding.GATE_FULL])
@pytest.mark.parametrize("normalise", [True, False])
def test_norm_after_the_residual(T, h, dtype, kind, normalise):
    x, y = _gauss((T, h), T + h, dtype, 2.0), _gauss((T, h), T + h + 1, dtype, 0.5)
    w = _gauss((h,), 2, dtype, 0.2, 1.0) if normalise and h % 2 == 0 else None
    wn = _gauss((h,), 3, dtype, 0.2, 1.0) if T % 2 else None
    gate = [None, _gauss((h,), 4, dtype), _gauss((T,), 4, dtype), _gauss((T, h), 4, dtype)][kind]
    out, codes, scale = binding.norm_residual_quant(x, y, w, 1e-6, gate=gate, gate_kind=kind if kind else None, residual_scale=0.9,
                                                    branch_scale=-1.2, normalise=normalise, next_weight=wn, next_eps=1e-5)
    a, b = (float(torch.tensor(v, dtype=F32)) for v in (0.9, -1.2))
    s = _want_sum(x, y, w, gate, kind, a, b, normalise, 1e-6)
    s.within(out, "sum")
    _check_codes(s, wn, 1e-5, True, codes, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,h", [(5, 1024), (400, 2048), (310, 7168), (320, 1031)])
def test_strides_and_the_stream_in_place(T, h, dtype):
    x, y = _gauss((T, h), 1, dtype), _gauss((T, h), 2, dtype)
    w = _gauss((h,), 3, dtype, 0.2, 1.0)
    want = binding.norm_residual_quant(x, y, w, 1e-6, next_weight=w)
    for pad, at in ((16, 16), (5, 3)):
        wide_x, wide_y = torch.zeros((T, h + pad), dtype=dtype, device=DEV), torch.zeros((T, h + pad), dtype=dtype, device=DEV)
        wide_c = torch.zeros((T, h + pad), dtype=torch.uint8, device=DEV)
        xs, ys, cs = wide_x[:, at:at + h], wide_y[:, at:at + h], wide_c.view(F8)[:, at:at + h]
        if at + h > h + pad:
            continue
        xs.copy_(x)
        ys.copy_(y)
        out, codes, scale = binding.norm_residual_quant(xs, ys, w, 1e-6, next_weight=w, out=xs, codes=cs)
        s = _want_sum(x, y, w, None, 0, 1.0, 1.0, True, 1e-6)
        s.within(out.contiguous(), "sum")
        _check_codes(s, w, 1e-6, True, codes, scale)
        assert (wide_c[:, :at] == 0).all() and (wide_c[:, at + h:] == 0).all() and (wide_x[:, :at] == 0).all()
    assert torch.equal(want[0], binding.norm_residual_quant(x, y, w, 1e-6, next_weight=w)[0])


@pytest.mark.parametrize("T", [4, 400])
def test_rows_of_every_size(T):
    """Rows of zeros, tiny and huge ones, infinities and NaN: each stays in its own row."""
    h = 1024
    x = _gauss((T, h), 5, F32)
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e30
    codes, scale = binding.norm_quant(x, None, 1e-6, normalise=False)
    _check_codes(Bounded(x), None, 1e-6, False, codes, scale)
    assert (codes[0].float() == 0).all() and torch.isfinite(scale).all()
    x[3] *= 3e38 / x[3].abs().max()
    codes, scale = binding.norm_quant(x, None, 1e-6, normalise=False)
    _check_codes(Bounded(x), None, 1e-6, False, codes, scale)
    clean = codes.float()
    x[1, 7], x[2, 9] = float("nan"), float("inf")
    codes, scale = binding.norm_quant(x, None, 1e-6)
    assert not torch.isfinite(scale[1:3]).any() and torch.isfinite(scale[0]) and torch.isfinite(scale[4:]).all()
    assert torch.equal(codes.float()[4:], clean[4:])


def test_equal_calls_give_equal_bits_and_a_captured_one_follows_its_inputs():
    T, h = 500, 4096
    s = {"x": _gauss((T, h), 1, BF16), "y": _gauss((T, h), 2, BF16), "w": _gauss((h,), 3, BF16)}

    def step():
        return binding.norm_residual_quant(s["x"], s["y"], s["w"], 1e-6, next_weight=s["w"])
    first = [t.clone() for t in step()]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, step()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    s["x"].copy_(_gauss((T, h), 9, BF16))
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(out, step()))


def test_no_tokens():
    x = torch.empty((0, 64), dtype=BF16, device=DEV)
    codes, scale = binding.norm_quant(x, None, 1e-6)
    assert codes.shape == (0, 64) and scale.shape == (0,)
    assert binding.norm_residual_quant(x, x.clone(), None, 1e-6)[1].shape == (0, 64)


def test_rows_beyond_32_bit_offsets():
    T, h = 2 ** 31 // 7168 + 5, 7168
    x = torch.zeros((T, h), dtype=BF16, device=DEV)
    x[-3:] = _gauss((3, h), 1, BF16)
    codes, scale = binding.norm_quant(x, None, 1e-6)
    _check_codes(Bounded(x[-3:]), None, 1e-6, True, codes[-3:], scale[-3:])
    out, codes, scale = binding.norm_residual_quant(x, codes.view(torch.uint8).to(BF16), None, 1e-6, normalise=False, out=x, codes=codes, scale=scale)
    assert torch.isfinite(scale).all()


def test_wrapper_refuses_what_does_not_fit():
    x, w = _gauss((6, 32), 1, BF16), _gauss((32,), 2, BF16)
    c, s = torch.empty((6, 32), dtype=F8, device=DEV), torch.empty(6, device=DEV)
    q, r = binding.norm_quant, binding.norm_residual_quant
    bad = [lambda: q(x.half(), w, 1e-6), lambda: q(x, w[:31], 1e-6), lambda: q(x, w, -1.0), lambda: q(x, w, 1e-6, codes=c[:5]),
           lambda: q(x, w, 1e-6, codes=c.view(torch.uint8)), lambda: q(x, w, 1e-6, scale=s[:5]), lambda: q(x, w, 1e-6, scale=s.to(BF16)),
           lambda: q(x.cpu(), None, 1e-6), lambda: r(x, x[:5], w, 1e-6), lambda: r(x, x, w, 1e-6, out=x), lambda: r(x, x.float(), w, 1e-6),
           lambda: r(x, x, w, 1e-6, next_weight=w.float()), lambda: r(x, x, w, 1e-6, gate=w[:30]), lambda: r(x, x, w, 1e-6, normalise=False),
           lambda: r(x, x, w, 1e-6, next_eps=float("nan"))]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()


# a block a row, value by value, and persistent blocks: without a sum, with one (four and two packs a thread), rows too wide for them
NOT_FINITE = [(1, 64), (5, 1024), (7, 1031), (400, 1031), (330, 2048), (310, 4096), (310, 7168), (300, 8192), (300, 16392)]


def _same(got, want, rows):
    return all(torch.equal(a[rows].view(torch.uint8), b[rows].view(torch.uint8)) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("T,h", NOT_FINITE)
def test_a_value_that_is_not_finite_shows_in_its_rows_scale(T, h, normalise, dtype):
    nan, inf = float("nan"), float("inf")
    x, w = _gauss((T, h), 1, dtype), _gauss((h,), 2, F32, 0.2, 1.0)
    w[h // 3] = 0.0
    clean = binding.norm_quant(x, w, 1e-6, normalise=normalise)
    assert torch.isfinite(clean[1]).all()
    for column, value in ((h - 1, nan), (0, inf), (h // 2, -inf), (h // 3, inf), (h // 3, nan)):  # under the gain of 0: 0 times it
        bad = x.clone()
        bad[T // 2, column] = value
        got = binding.norm_quant(bad, w, 1e-6, normalise=normalise)
        rest = [t for t in range(T) if t != T // 2]
        assert not torch.isfinite(got[1][T // 2]) and _same(got, clean, rest), (column, value)
    x[T // 2] = nan
    assert torch.isnan(binding.norm_quant(x, None, 1e-6, normalise=normalise)[1][T // 2])
    w[h // 2] = nan
    assert not torch.isfinite(binding.norm_quant(clean[0].to(dtype), w, 1e-6, normalise=normalise)[1]).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", [binding.GATE_NONE, binding.GATE_TOKEN, binding.GATE_FULL])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("T,h", NOT_FINITE)
def test_a_value_that_is_not_finite_shows_in_the_scale_after_the_residual(T, h, normalise, kind, dtype):
    nan, inf = float("nan"), float("inf")
    x, y = _gauss((T, h), 1, dtype), _gauss((T, h), 2, dtype)
    wn = _gauss((h,), 3, dtype, 0.2, 1.0)
    wn[h // 3] = 0.0
    gate = [None, None, _gauss((T,), 4, dtype), _gauss((T, h), 4, dtype)][kind]

    def call(x, y, gate, wn):
        return binding.norm_residual_quant(x, y, None, 1e-6, gate=gate, gate_kind=kind if kind else None, normalise=normalise, next_weight=wn)[1:]

    clean, rest = call(x, y, gate, wn), [t for t in range(T) if t != T // 2]
    assert torch.isfinite(clean[1]).all()
    for which, column, value in ((0, h - 1, nan), (0, h // 3, inf), (1, 0, nan), (1, h // 2, inf), (2, 0, nan)):
        args = [x.clone(), y.clone(), gate if gate is None else gate.clone()]
        if args[which] is None:
            continue
        at = (T // 2,) if args[which].dim() == 1 else (T // 2, column)
        args[which][at] = value
        got = call(*args, wn)
        assert not torch.isfinite(got[1][T // 2]) and _same(got, clean, rest), (which, column, value)
    wn[0] = nan
    assert not torch.isfinite(call(x, y, gate, wn)[1]).any()
