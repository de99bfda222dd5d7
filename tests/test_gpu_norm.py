"""Norms around a block and their gradients against plain definitions with rigorous fp32 bounds."""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests.bounds import Bounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def _gauss(shape, dtype, seed, scale=1.0, mean=0.0, layout="dense"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if layout == "dense" or len(shape) == 1:
        return (torch.randn(shape, generator=g, device=DEV) * scale + mean).to(dtype)
    pad, at = (16, 8) if layout == "strided" else (7, 3)
    wide = (torch.randn((shape[0], shape[1] + pad), generator=g, device=DEV) * scale + mean).to(dtype)
    return wide[:, at:at + shape[1]]


def _inv(v, eps):
    return ((v * v).sum(1, keepdim=True) * Bounded(1.0 / v.v.shape[1]) + Bounded(eps)).rsqrt()


def _unit_grad(v, r, d):
    """r d - v r^3 mean(d v)."""
    mean = (d * v).sum(1, keepdim=True) * Bounded(1.0 / v.v.shape[1])
    return r * d - v * (r * r * r * mean)


# rows of one value up to wide ones; sizes around 8-value packs, warps and blocks of them; more rows than thread blocks
SHAPES = [(1, 1), (1, 7168), (3, 8), (5, 72), (2, 1027), (300, 64), (128, 4096), (33, 2056), (601, 520), (17, 7168),
          (4, 16384), (3, 16392), (2, 40000), (7, 9001)]


@pytest.mark.parametrize("layout", ["dense", "strided", "odd"])
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("T,h", SHAPES)
def test_norm_and_its_gradient(T, h, dtype, wdtype, layout):
    eps = 1e-6
    x = _gauss((T, h), dtype, 1, 2.0, layout=layout)
    w = _gauss((h,), wdtype, 2, 0.3, 1.0)
    x[T // 2] = 0                                             # a row of zeros
    X, W = Bounded(x), Bounded(w)
    r = _inv(X, eps)
    out = binding.norm(x, w, eps, out=_gauss((T, h), dtype, 3, layout=layout))
    (X * r * W).within(out, "norm")
    du, dadd = _gauss((T, h), dtype, 4, layout=layout), _gauss((T, h), dtype, 5, layout=layout)
    dx, dw = binding.norm_backward(x, w, eps, du, dx=_gauss((T, h), dtype, 6, layout=layout))
    D = Bounded(du)
    want = _unit_grad(X, r, D * W)
    want.within(dx, "dx")
    (D * X * r).sum(0).within(dw, "dw")
    dx2, dw2 = binding.norm_backward(x, w, eps, du, dadd=dadd)
    (want + Bounded(dadd)).within(dx2, "dx + dadd")
    assert torch.equal(dw, dw2)
    ones, _ = binding.norm_backward(x, None, eps, du)
    _unit_grad(X, r, D).within(ones, "dx without a gain")


def _block(x, y, w, wn, gate, kind, a, b, eps, next_eps, normalise):
    """s, branch and the inverse rms values of the definition, with bounds."""
    X, Y = Bounded(x), Bounded(y)
    W = Bounded(w) if w is not None else Bounded(1.0)
    ry = _inv(Y, eps) if normalise else Bounded(1.0)
    branch = Y * ry * W if normalise else Y * W
    G = Bounded(1.0) if gate is None else Bounded(gate)
    if kind == binding.GATE_TOKEN:
        G = Bounded(gate[:, None])
    s = Bounded(a) * X + Bounded(b) * G * branch
    return X, Y, W, ry, branch, G, s, _inv(s, next_eps)


CASES = [(1, 1, "none"), (1, 4096, "channel"), (5, 72, "token"), (2, 1027, "full"), (300, 64, "channel"), (33, 2056, "token"),
         (601, 520, "full"), (17, 7168, "channel"), (3, 16392, "channel"), (2, 40000, "full"), (7, 9001, "token"),
         (64, 64, "token"), (64, 64, "channel"), (40, 8192, "full"), (9, 12288, "channel")]
KINDS = {"none": None, "channel": binding.GATE_CHANNEL, "token": binding.GATE_TOKEN, "full": binding.GATE_FULL}


@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("normalise,next_norm", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("T,h,gate_kind", CASES)
def test_norm_residual_and_its_gradient(T, h, gate_kind, dtype, wdtype, normalise, next_norm, layout):
    # fp32 scales, so that the definition multiplies by the same numbers
    a, b, eps, next_eps = 0.75, 1.5, 2.0 ** -20, 2.0 ** -17
    kind = KINDS[gate_kind]
    x, y = _gauss((T, h), dtype, 1, 2.0, layout=layout), _gauss((T, h), dtype, 2, 0.5, layout=layout)
    w = _gauss((h,), wdtype, 3, 0.3, 1.0) if normalise else None
    wn = _gauss((h,), wdtype, 4, 0.3, 1.0) if next_norm else None
    shape = {"none": None, "channel": (h,), "token": (T,), "full": (T, h)}[gate_kind]
    gate = None if shape is None else _gauss(shape, dtype, 5, 0.5, 0.3, layout=layout)
    kw = dict(gate=gate, residual_scale=a, branch_scale=b, normalise=normalise, next_weight=wn, next_eps=next_eps,
              gate_kind=kind)
    X, Y, W, ry, branch, G, s, ro = _block(x, y, w, wn, gate, kind, a, b, eps, next_eps, normalise)
    out, u = binding.norm_residual(x, y, w, eps, next_norm=next_norm, **kw)
    s.within(out, "out")
    if next_norm:
        (s * ro * Bounded(wn)).within(u, "next")
    else:
        assert u is None
    place = x.clone()
    binding.norm_residual(place, y, w, eps, next_norm=next_norm, out=place, **kw)          # the stream in place
    assert torch.equal(place, out)

    dout = _gauss((T, h), dtype, 6, layout=layout)
    du = _gauss((T, h), dtype, 7, layout=layout) if next_norm else None
    dx, dy, dgate, dw, dn = binding.norm_residual_backward(x, y, w, eps, dout, du=du, **kw)
    D = Bounded(dout)
    if next_norm:
        D = D + _unit_grad(s, ro, Bounded(du) * Bounded(wn))
        (Bounded(du) * s * ro).sum(0).within(dn, "dnext_weight")
    else:
        assert dn is None
    (Bounded(a) * D).within(dx, "dx")
    dv = Bounded(b) * G * D
    dv = dv * Bounded(torch.ones_like(D.v))
    if normalise:
        _unit_grad(Y, ry, dv * W).within(dy, "dy")
        (dv * Y * ry).sum(0).within(dw, "dweight")
    else:
        dv.within(dy, "dy")
        assert dw is None
    dg = Bounded(b) * D * branch
    if kind is None:
        assert dgate is None
    elif kind == binding.GATE_CHANNEL:
        dg.sum(0).within(dgate, "dgate")
    elif kind == binding.GATE_TOKEN:
        dg.sum(1).within(dgate, "dgate")
    else:
        dg.within(dgate, "dgate")


def test_gradients_against_differences():
    """The gradients along a random direction against central differences of the definition in 64 bits (step 1e-4:
    truncation and rounding below 1e-6 of the sums' size for these smooth functions of order one)."""
    T, h, a, b, eps = 13, 96, 0.75, 1.5, 1e-6
    leaves = {"x": (T, h), "y": (T, h), "w": (h,), "wn": (h,), "gate": (h,)}
    v = {n: _gauss(s, F32, i, 0.5, 1.0) for i, (n, s) in enumerate(leaves.items())}
    along = {n: _gauss(s, F32, 20 + i).double() for i, (n, s) in enumerate(leaves.items())}
    dout, du = _gauss((T, h), F32, 40), _gauss((T, h), F32, 41)

    def loss(step):
        p = {n: v[n].double() + step * along[n] for n in leaves}
        unit = lambda m: m / torch.sqrt((m * m).mean(1, keepdim=True) + eps)  # noqa: E731
        s = a * p["x"] + b * p["gate"] * unit(p["y"]) * p["w"]
        return (s * dout.double()).sum() + (unit(s) * p["wn"] * du.double()).sum()

    difference = (loss(1e-4) - loss(-1e-4)) / 2e-4
    dx, dy, dgate, dw, dn = binding.norm_residual_backward(v["x"], v["y"], v["w"], eps, dout, gate=v["gate"], residual_scale=a,
                                                           branch_scale=b, next_weight=v["wn"], du=du)
    parts = [(dx, "x"), (dy, "y"), (dw, "w"), (dn, "wn"), (dgate, "gate")]
    got = sum((g.double() * along[n]).sum() for g, n in parts)
    size = sum((g.double().abs() * along[n].abs()).sum() for g, n in parts)
    assert abs(got - difference) <= 1e-5 * size


def test_no_tokens():
    x = torch.empty((0, 64), dtype=BF16, device=DEV)
    w = _gauss((64,), F32, 1)
    assert binding.norm(x, w, 1e-6).shape == (0, 64)
    _, dw = binding.norm_backward(x, w, 1e-6, x)
    assert (dw == 0).all()
    out, u = binding.norm_residual(x, x, w, 1e-6, next_weight=w)
    assert out.shape == u.shape == (0, 64)
    _, _, dgate, dw, dn = binding.norm_residual_backward(x, x, w, 1e-6, x, gate=_gauss((64,), BF16, 2), next_weight=w, du=x)
    assert (dgate == 0).all() and (dw == 0).all() and (dn == 0).all()


def test_infinities_and_nan_stay_in_their_row():
    T, h = 5, 4096
    x, y, w = _gauss((T, h), BF16, 1), _gauss((T, h), BF16, 2), _gauss((h,), BF16, 3)
    clean_u, (clean_out, clean_n) = binding.norm(x, w, 1e-6), binding.norm_residual(x, y, w, 1e-6, next_weight=w)
    x2, y2 = x.clone(), y.clone()
    x2[1, 7], y2[3, 9] = float("inf"), float("nan")
    u, (out, n) = binding.norm(x2, w, 1e-6), binding.norm_residual(x2, y2, w, 1e-6, next_weight=w)
    keep = [0, 2, 4]
    assert torch.equal(u[keep], clean_u[keep]) and torch.equal(out[keep], clean_out[keep]) and torch.equal(n[keep], clean_n[keep])
    assert torch.isnan(u[1, 7]) and torch.isinf(out[1, 7]) and torch.isnan(out[3]).all() and torch.isnan(n[3]).all()


def test_gradient_in_place_of_the_residual_gradient():
    x, w, du, dadd = (_gauss(s, BF16, i) for i, s in enumerate([(50, 520), (520,), (50, 520), (50, 520)]))
    want, _ = binding.norm_backward(x, w, 1e-6, du, dadd=dadd)
    got, _ = binding.norm_backward(x, w, 1e-6, du, dadd=dadd, dx=dadd)
    assert got is dadd and torch.equal(got, want)


def test_captured_and_on_two_streams():
    """A training step's norm calls captured once each for two sets of tensors, replayed side by side on new data."""
    def step(s):
        u = binding.norm(s["x"], s["w"], 1e-6)
        out, n = binding.norm_residual(s["x"], s["y"], s["w"], 1e-6, gate=s["g"], next_weight=s["w"])
        grads = binding.norm_residual_backward(s["x"], s["y"], s["w"], 1e-6, s["d"], gate=s["g"], next_weight=s["w"], du=s["y"])
        return (u, out, n) + grads + binding.norm_backward(s["x"], s["w"], 1e-6, s["d"], dadd=grads[0])

    def fill(seed):
        return {"x": _gauss((700, 1024), BF16, seed), "y": _gauss((700, 1024), BF16, seed + 1), "d": _gauss((700, 1024), BF16, seed + 2),
                "w": _gauss((1024,), BF16, seed + 3, 0.2, 1.0), "g": _gauss((1024,), BF16, seed + 4)}

    states, graphs, outs = [fill(0), fill(10)], [], []
    for s in states:
        step(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    for i, s in enumerate(states):
        for n, t in fill(50 + 10 * i).items():
            s[n].copy_(t)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s, got in zip(states, outs):
        for a, b in zip(got, step(s)):
            assert torch.equal(a, b)


def test_wrapper_refuses_what_does_not_fit():
    x, w = _gauss((4, 64), BF16, 1), _gauss((64,), BF16, 2)
    square = _gauss((64, 64), BF16, 3)
    bad = [lambda: binding.norm(x.half(), w, 1e-6), lambda: binding.norm(x, w[:63], 1e-6), lambda: binding.norm(x, w, -1.0),
           lambda: binding.norm(x, w.half(), 1e-6), lambda: binding.norm(x.cpu(), w, 1e-6), lambda: binding.norm(x.t(), w, 1e-6),
           lambda: binding.norm(x, w, float("nan")), lambda: binding.norm_backward(x, w, 1e-6, x.float()),
           lambda: binding.norm_residual(x, x[:3], w, 1e-6), lambda: binding.norm_residual(x, x.clone(), w, 1e-6, normalise=False),
           lambda: binding.norm_residual(x, x.clone(), w, 1e-6, gate=w[:5]),
           lambda: binding.norm_residual(x, x.clone(), w, 1e-6, next_weight=w.float()),
           lambda: binding.norm_residual(x, x, w, 1e-6, out=x), lambda: binding.norm_residual(square, square.clone(), w, 1e-6, gate=w),
           lambda: binding.norm_residual(x, x.clone(), w, 1e-6, residual_scale=float("nan")),
           lambda: binding.norm_residual_backward(x, x.clone(), w, 1e-6, x.clone(), next_weight=w),
           lambda: binding.norm_backward(x, w, 1e-6, x.clone(), dx=x)]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()


def test_rows_beyond_32_bit_offsets():
    """Over 2^31 values: the last rows of the norm and of its gradient."""
    T, h = 300032, 7168
    assert T * h > 2 ** 31
    x = torch.empty((T, h), dtype=BF16, device=DEV)
    x[:-40] = 1
    x[-40:] = _gauss((40, h), BF16, 1)
    w = _gauss((h,), BF16, 2, 0.3, 1.0)
    X, W = Bounded(x[-40:]), Bounded(w)
    r = _inv(X, 1e-6)
    (X * r * W).within(binding.norm(x, w, 1e-6)[-40:], "norm")
    dx, _ = binding.norm_backward(x, w, 1e-6, x)
    _unit_grad(X, r, X * W).within(dx[-40:], "dx")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,h", [(5, 1024), (3, 1027), (2, 16392)])
@pytest.mark.parametrize("x_size,y_size,eps", [(1e15, 1.0, 1e-6), (1.0, 1e15, 1e-6), (1e15, 1e15, 1e-6), (1.0, 1e-14, 0.0), (1e-14, 1.0, 0.0)])
def test_gradients_of_very_large_and_very_small_rows(x_size, y_size, eps, T, h, dtype):
    """Rows whose inverse rms cubed no fp32 number holds, but whose gradients one does."""
    x, y = _gauss((T, h), dtype, 1, x_size), _gauss((T, h), dtype, 2, y_size)
    w, wn, gate = _gauss((h,), dtype, 3, 0.3, 1.0), _gauss((h,), dtype, 4, 0.3, 1.0), _gauss((T,), dtype, 5, 0.3, 1.0)
    dout, du = _gauss((T, h), dtype, 6), _gauss((T, h), dtype, 7)
    X, W, D = Bounded(x), Bounded(w), Bounded(du)
    r = _inv(X, eps)
    (X * r * W).within(binding.norm(x, w, eps), "norm")
    dx, dw = binding.norm_backward(x, w, eps, du)
    _unit_grad(X, r, D * W).within(dx, "dx")
    (D * X * r).sum(0).within(dw, "dw")
    kind = binding.GATE_TOKEN
    X, Y, W, ry, branch, G, s, ro = _block(x, y, w, wn, gate, kind, 0.75, 1.5, eps, eps, True)
    dx, dy, dgate, dw, dn = binding.norm_residual_backward(x, y, w, eps, dout, gate=gate, residual_scale=0.75, branch_scale=1.5,
                                                           next_weight=wn, du=du, gate_kind=kind)
    total = Bounded(dout) + _unit_grad(s, ro, Bounded(du) * Bounded(wn))
    (Bounded(0.75) * total).within(dx, "dx of the block")
    dv = Bounded(1.5) * G * total
    _unit_grad(Y, ry, dv * W).within(dy, "dy")
    (dv * Y * ry).sum(0).within(dw, "dweight")
    (Bounded(du) * s * ro).sum(0).within(dn, "dnext_weight")
    (Bounded(1.5) * total * branch).sum(1).within(dgate, "dgate")


@pytest.mark.parametrize("T,h", [(6, 64), (64, 64), (1, 8), (5, 1)])
def test_a_column_of_token_gates(T, h):
    """[T, 1], as a projection with one output makes it, is the gate [T]; its gradient comes in its shape."""
    x, y, w, dout = _gauss((T, h), BF16, 1), _gauss((T, h), BF16, 2), _gauss((h,), BF16, 3, 0.3, 1.0), _gauss((T, h), BF16, 4)
    gate = _gauss((T, 1), BF16, 5)
    flat, column = dict(gate=gate[:, 0].contiguous(), gate_kind=binding.GATE_TOKEN), dict(gate=gate, gate_kind=binding.GATE_TOKEN)
    for kw in (column, dict(gate=gate)) if h > 1 else (column,):
        for a, b in zip(binding.norm_residual(x, y, w, 1e-6, next_weight=w, **kw), binding.norm_residual(x, y, w, 1e-6, next_weight=w, **flat)):
            assert torch.equal(a, b)
        got = binding.norm_residual_backward(x, y, w, 1e-6, dout, next_weight=w, du=y, **kw)
        want = binding.norm_residual_backward(x, y, w, 1e-6, dout, next_weight=w, du=y, **flat)
        assert got[2].shape == (T, 1) and got[2].dtype == F32 and want[2].shape == (T,)
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a[:, 0] if i == 2 else a, b)
    wide = _gauss((T, 2), BF16, 6)[:, :1]                       # not contiguous
    if T > 1:
        with pytest.raises(binding.DeaMoEError):
            binding.norm_residual(x, y, w, 1e-6, gate=wide, gate_kind=binding.GATE_TOKEN)


# Blocks of the gradient kernels that walk several rows each: the ring of rows ahead holds 4 (7168 bf16), 3 (7168 bf16 with a
# full gate, 4096 and 1024 bf16), 2 (7168 fp32) or 1 (7168 fp32 with a full gate, 4096 and 1024 fp32); 1027 is read value by
# value; 9001 goes through the form for any width.
MANY = [(500, 7168), (950, 4096), (3700, 1024), (2300, 1027), (900, 9001), (4000, 24)]


def _rows_a_block(T, h):
    return T * 12 * h / binding.lib().deamoe_norm_workspace(T, h)    # the workspace holds three rows of sums a block


@pytest.mark.parametrize("dtype,wdtype", [(BF16, F32), (F32, F32)])
@pytest.mark.parametrize("T,h", MANY)
def test_norm_gradient_with_many_rows_a_block(T, h, dtype, wdtype):
    assert _rows_a_block(T, h) >= 3
    eps = 1e-6
    x, du, dadd = (_gauss((T, h), dtype, i, 1.0 + i) for i in range(3))
    w = _gauss((h,), wdtype, 9, 0.3, 1.0)
    X, W, D = Bounded(x), Bounded(w), Bounded(du)
    r = _inv(X, eps)
    want, sums = _unit_grad(X, r, D * W), (D * X * r).sum(0)
    for add in (None, dadd):
        dx, dw = binding.norm_backward(x, w, eps, du, dadd=add)
        (want if add is None else want + Bounded(add)).within(dx, "dx")
        sums.within(dw, "dw")
        again = binding.norm_backward(x, w, eps, du, dadd=add)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("normalise,next_norm", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("gate_kind", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,h", MANY)
def test_residual_gradient_with_many_rows_a_block(T, h, dtype, gate_kind, normalise, next_norm):
    assert _rows_a_block(T, h) >= 3
    a, b, eps, next_eps = 0.75, 1.5, 2.0 ** -20, 2.0 ** -17
    kind = KINDS[gate_kind]
    shape = {"none": None, "channel": (h,), "token": (T,), "full": (T, h)}[gate_kind]
    x, y, dout = (_gauss((T, h), dtype, i, 0.5 + i) for i in range(3))
    du = _gauss((T, h), dtype, 3) if next_norm else None
    w = _gauss((h,), F32, 4, 0.3, 1.0) if normalise else None
    wn = _gauss((h,), F32, 5, 0.3, 1.0) if next_norm else None
    gate = None if shape is None else _gauss(shape, dtype, 6, 0.5, 0.3)
    X, Y, W, ry, branch, G, s, ro = _block(x, y, w, wn, gate, kind, a, b, eps, next_eps, normalise)

    def call():
        return binding.norm_residual_backward(x, y, w, eps, dout, gate=gate, residual_scale=a, branch_scale=b, normalise=normalise,
                                              next_weight=wn, next_eps=next_eps, du=du, gate_kind=kind)

    dx, dy, dgate, dw, dn = got = call()
    D = Bounded(dout)
    if next_norm:
        D = D + _unit_grad(s, ro, Bounded(du) * Bounded(wn))
        (Bounded(du) * s * ro).sum(0).within(dn, "dnext_weight")
    (Bounded(a) * D).within(dx, "dx")
    dv = Bounded(b) * G * D
    if normalise:
        _unit_grad(Y, ry, dv * W).within(dy, "dy")
        (dv * Y * ry).sum(0).within(dw, "dweight")
    else:
        dv.within(dy, "dy")
    if kind is not None:
        dg = Bounded(b) * D * branch
        (dg if kind == binding.GATE_FULL else dg.sum(0 if kind == binding.GATE_CHANNEL else 1)).within(dgate, "dgate")
    for p, q in zip(got, call()):
        assert p is None and q is None or torch.equal(p, q)
