"""Matrix products with bias, activation and residual, from bf16 and from 8-bit rows, and their gradients, against their
definition in 64 bits."""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests import product_bounds as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
NONE, SILU, GELU = binding.SIGMA_NONE, binding.SIGMA_SILU, binding.SIGMA_GELU


def _g(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _gauss(shape, seed, scale=1.0, dtype=BF16):
    return (torch.randn(shape, generator=_g(seed), device=DEV) * scale).to(dtype)


def _case(T, K, N, kind, seed, bias=None, residual=False):
    c = {"x": _gauss((T, K), seed), "w": _gauss((N, K), seed + 1, K ** -0.5), "xs": None, "ws": None}
    if kind == "e4m3":
        for a, b in (("x", "xs"), ("w", "ws")):
            v = c[a].float()
            c[b] = v.abs().amax(1).clamp(min=1e-6) / 448
            c[a] = (v / c[b][:, None]).to(F8)
    c["bias"] = None if bias is None else _gauss((N,), seed + 2, 0.5, bias)
    c["residual"] = _gauss((T, N), seed + 3) if residual else None
    return c


def _call(c, act=NONE, out=None):
    return binding.product(c["x"], c["w"], bias=c["bias"], act=act, residual=c["residual"], x_scale=c["xs"], weight_scale=c["ws"], out=out)


def _want(c, act):
    x, w = c["x"].double(), c["w"].double()
    z, e = pb.dot(x, None, w, None)
    if c["xs"] is not None:
        s = c["xs"].double()[:, None] * c["ws"].double()[None, :]
        z, e = pb.times(z, e, s, s.abs() * pb.UNIT)
    if c["bias"] is not None:
        z, e = pb.plus(z, e, c["bias"].double()[None, :], torch.zeros_like(z))
    z, e = pb.act(act, z, e)
    if c["residual"] is not None:
        z, e = pb.plus(z, e, c["residual"].double(), torch.zeros_like(z))
    return z, e


# one to 300 tokens around the forms' limits (8, 16, 64, 128, 256), odd and ragged matrices, one value to long rows
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(1, 16, 1), (1, 7168, 33), (3, 48, 17), (8, 128, 100), (9, 272, 64), (16, 1040, 520), (17, 64, 8), (17, 4096, 40),
                                   (31, 160, 1003), (64, 7168, 256), (65, 144, 257), (100, 3104, 300), (129, 2048, 999), (256, 32, 512),
                                   (257, 512, 130), (300, 1008, 264), (1000, 80, 72)])
@pytest.mark.parametrize("act,bias,residual", [(NONE, None, False), (SILU, torch.float32, True), (GELU, BF16, False), (NONE, BF16, True)])
def test_product(T, K, N, kind, act, bias, residual):
    c = _case(T, K, N, kind, T + K + N, bias, residual)
    pb.check(_call(c, act), *_want(c, act))
    assert binding.operator_status() == binding.OK


@pytest.mark.parametrize("act,bias", [(NONE, None), (NONE, torch.float32), (SILU, BF16), (GELU, None), (GELU, torch.float32), (SILU, None)])
@pytest.mark.parametrize("T,K,N", [(1, 8, 8), (1, 520, 64), (7, 72, 40), (16, 16, 256), (33, 264, 136), (63, 128, 128), (64, 1096, 8), (65, 8, 520),
                                   (200, 200, 344), (257, 512, 72), (700, 264, 520), (2100, 136, 264)])
def test_gradients(T, K, N, act, bias):
    c = _case(T, K, N, "bf16", T + K + N, bias)
    dout = _gauss((T, N), 9)
    dx, dw, db = binding.product_backward(c["x"], c["w"], dout, bias=c["bias"], act=act)
    x, w, d = c["x"].double(), c["w"].double(), dout.double()
    dz, e, eb = d, None, torch.zeros_like(d)
    if act != NONE:
        z, ez = pb.dot(x, None, w, None)
        if c["bias"] is not None:
            z, ez = pb.plus(z, ez, c["bias"].double()[None, :], torch.zeros_like(z))
        dz, eb = pb.times(d, torch.zeros_like(d), *pb.act_grad(act, z, ez))
        dz, e = pb.to_bf16(dz, eb)
    pb.check(dx, *pb.dot(dz, e, w.T, None), "dx")
    pb.check(dw, *pb.dot(dz.T, None if e is None else e.T, x.T, None), "dweight")
    assert (db is None) == (bias is None)
    if db is not None:  # fp32 sums of the unrounded dz: one rounding a row
        pb.check(db, dz.sum(0), eb.sum(0) + (T + 8) * 2.0 ** -24 * (dz.abs() + eb).sum(0), "dbias")


def test_gradients_against_differences():
    """As for the feed-forward blocks: central differences of the definition in 64 bits, steps of 2^-10."""
    T, K, N = 37, 72, 48
    c = _case(T, K, N, "bf16", 3, torch.float32)
    dout = _gauss((T, N), 4)
    for act, fn in ((NONE, lambda z: z), (SILU, torch.nn.functional.silu), (GELU, torch.nn.functional.gelu)):
        leaves = [c["x"].double(), c["w"].double(), c["bias"].double()]
        loss = lambda x, w, b: (fn(x @ w.T + b) * dout.double()).sum()  # noqa: E731
        got = binding.product_backward(c["x"], c["w"], dout, bias=c["bias"], act=act)
        for i, g in enumerate(got):
            D = torch.randn(leaves[i].shape, generator=_g(20 + i), device=DEV, dtype=torch.float64)
            D /= D.norm()
            up, down = list(leaves), list(leaves)
            up[i], down[i] = leaves[i] + 2.0 ** -10 * D, leaves[i] - 2.0 ** -10 * D
            want = (loss(*up) - loss(*down)) / 2.0 ** -9
            # dz and the result rounded to bf16: 2^-8 of their terms' sizes, each direction's terms independent of D
            size = (g.double().abs() * D.abs()).sum() * 2 + g.double().norm()
            assert abs((g.double() * D).sum() - want) <= (2 * pb.BF16_HALF + 1e-4) * size, (act, i)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T", [5, 40, 300])
def test_strides_are_followed_and_out_may_be_the_residual(T, kind):
    K, N = 144, 77
    c = _case(T, K, N, kind, 5, BF16, True)
    plain = _call(c, SILU)
    wide_x = torch.zeros((T, K + 32), dtype=c["x"].dtype, device=DEV)
    wide_x[:, 16:16 + K] = c["x"]
    room = _gauss((T, N + 11), 6)
    for at in (0, 3, 8):                                   # outputs on and off 16-byte boundaries
        r = room.clone()
        r[:, at:at + N] = c["residual"]
        kept = r.clone()
        s = dict(c, x=wide_x[:, 16:16 + K], residual=r[:, at:at + N])
        assert torch.equal(_call(s, SILU, out=r[:, at:at + N]), plain)
        assert torch.equal(r[:, :at], kept[:, :at]) and torch.equal(r[:, at + N:], kept[:, at + N:])


def test_gradient_strides_are_followed():
    T, K, N = 70, 136, 72
    c = _case(T, K, N, "bf16", 7, BF16)
    dout = _gauss((T, N), 8)
    want = binding.product_backward(c["x"], c["w"], dout, bias=c["bias"], act=GELU)
    x, d, dx = (torch.zeros((T, n + 24), dtype=BF16, device=DEV) for n in (K, N, K))
    x[:, 8:8 + K], d[:, 16:16 + N] = c["x"], dout
    got = binding.product_backward(x[:, 8:8 + K], c["w"], d[:, 16:16 + N], bias=c["bias"], act=GELU, dx=dx[:, 8:8 + K])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (dx[:, :8] == 0).all() and (dx[:, 8 + K:] == 0).all()
    assert torch.equal(dx[:, 8:8 + K], want[0])


@pytest.mark.parametrize("T", [4, 30, 300])
def test_values_that_are_not_finite_stay_with_their_row(T):
    c = _case(T, 64, 40, "bf16", 9, BF16)
    clean = _call(c, GELU)
    c["x"][1, 5], c["x"][2, 7] = float("nan"), float("inf")
    got = _call(c, NONE)
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()
    got = _call(c, GELU)
    rest = [0] + list(range(3, T))
    assert torch.isnan(got[1]).all() and torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("T", [3, 50])
def test_ends_of_the_eight_bit_range(T):
    """Codes of +-448 and subnormal codes, scales far from one: products are exact sums, rounded once."""
    K, N = 128, 24
    g = _g(10)
    x = torch.randint(0, 127, (T, K), generator=g, device=DEV, dtype=torch.uint8)
    w = torch.randint(0, 127, (N, K), generator=g, device=DEV, dtype=torch.uint8)
    x[:, ::3] |= 128
    x[:, :8], w[:, :8] = 126, 1                            # 448 and 2^-9
    x, w = x.view(F8), w.view(F8)
    xs = torch.logspace(-12, 12, T, device=DEV)
    ws = torch.logspace(-10, 10, N, device=DEV)
    c = {"x": x, "w": w, "xs": xs, "ws": ws, "bias": None, "residual": None}
    pb.check(_call(c), *_want(c, NONE))


def test_equal_calls_give_equal_bits():
    for T in (6, 40, 700):
        c = _case(T, 2048, 520, "bf16", 11, BF16, True)
        dout = _gauss((T, 520), 12)
        first = [_call(c, SILU), *binding.product_backward(c["x"], c["w"], dout, bias=c["bias"], act=SILU)]
        for _ in range(4):
            again = [_call(c, SILU), *binding.product_backward(c["x"], c["w"], dout, bias=c["bias"], act=SILU)]
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_no_tokens():
    w = _gauss((24, 16), 1)
    x, d = torch.empty((0, 16), dtype=BF16, device=DEV), torch.empty((0, 24), dtype=BF16, device=DEV)
    assert binding.product(x, w).shape == (0, 24)
    dx, dw, db = binding.product_backward(x, w, d, bias=torch.zeros(24, device=DEV), act=SILU)
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()


def test_captured_calls_on_two_streams_share_nothing():
    K, N = 1032, 264
    w, bias = _gauss((N, K), 1, K ** -0.5), _gauss((N,), 2)

    def step(s):
        return (binding.product(s["x"], w, bias=bias, act=GELU), binding.product(s["x"][:7], w),
                *binding.product_backward(s["x"], w, s["d"], bias=bias, act=GELU))

    states = [{"x": _gauss((90, K), i), "d": _gauss((90, N), i + 9)} for i in (1, 2)]
    graphs, outs = [], []
    for s in states:
        step(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    for i, s in enumerate(states):
        s["x"].copy_(_gauss((90, K), 20 + i))
        s["d"].copy_(_gauss((90, N), 30 + i))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s, got in zip(states, outs):
        assert all(torch.equal(a, b) for a, b in zip(got, step(s)))


def test_outputs_beyond_32_bit_offsets():
    T, K, N = 70000, 16, 32768
    c = _case(T, K, N, "bf16", 13)
    out = _call(c)
    assert out.numel() > 2 ** 31
    for rows in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        pb.check(out[rows], *pb.dot(c["x"][rows].double(), None, c["w"].double(), None))


def test_wrapper_refuses_what_does_not_fit():
    x, w = _gauss((6, 32), 1), _gauss((24, 32), 2)
    x8, w8, s = x.to(F8), w.to(F8), torch.ones(6, device=DEV)
    t = torch.ones(24, device=DEV)
    p, b = binding.product, binding.product_backward
    d = _gauss((6, 24), 3)
    bad = [lambda: p(x.float(), w), lambda: p(x, w.float()), lambda: p(x, w[:, :16]), lambda: p(x, w, act=binding.SIGMA_RMSNORM),
           lambda: p(x, w, bias=t[:23]), lambda: p(x, w, bias=t.half()), lambda: p(x, w, residual=x), lambda: p(x, w, residual=d.float()),
           lambda: p(x, w, x_scale=s), lambda: p(x8, w8), lambda: p(x8, w8, x_scale=s), lambda: p(x8, w, x_scale=s, weight_scale=t),
           lambda: p(x8, w8, x_scale=s.to(BF16), weight_scale=t), lambda: p(x, w.cpu()), lambda: p(x[:, 1:25], w[:, :24].contiguous()),
           lambda: p(x[:, :28], w[:, :28].contiguous()), lambda: p(x8[:, :24], w8[:, :24].contiguous(), x_scale=s, weight_scale=t),
           lambda: p(x, w, out=d[:5]), lambda: b(x8, w8, d), lambda: b(x, w, d[:, :16]), lambda: b(x, w, x), lambda: b(x, w, d, dx=x),
           lambda: b(x, w, d, dweight=w), lambda: b(x, w[:20], d[:, :20].contiguous()), lambda: b(x, w, d, act=7)]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()


def test_bias_gradient_of_millions_of_tokens():
    """More rows than a grid's smaller sides hold blocks of them."""
    T, K, N = 65536 * 64 + 77, 8, 8
    x, w, d = _gauss((T, K), 1), _gauss((N, K), 2), _gauss((T, N), 3)
    dx, dw, db = binding.product_backward(x, w, d, bias=torch.zeros(N, device=DEV))
    for rows in (slice(0, 50), slice(T - 50, T)):
        pb.check(dx[rows], *pb.dot(d[rows].double(), None, w.double().T, None))
    pb.check(db, d.double().sum(0), (T + 8) * 2.0 ** -24 * d.double().abs().sum(0))
    pb.check(dw, *pb.dot(d.double().T, None, x.double().T, None))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(300, 144, 72), (2100, 264, 1040), (40, 2048, 136)])
def test_residual_and_out_on_different_boundaries(T, K, N, kind):
    """An aligned out with a residual off 16-byte boundaries, and the other way round; also rows of whole pieces with a stride that is not."""
    K = K // 16 * 16
    c = _case(T, K, N, kind, 21, BF16, True)
    plain = _call(c, GELU)
    for at, pad in ((0, 16), (3, 16), (8, 16), (0, 3)):
        room = torch.zeros((T, N + pad), dtype=BF16, device=DEV)
        room[:, at:at + N] = c["residual"]
        s = dict(c, residual=room[:, at:at + N])
        assert torch.equal(_call(s, GELU), plain)
        out = torch.full((T, N + pad), 3.0, dtype=BF16, device=DEV)
        assert torch.equal(_call(c, GELU, out=out[:, at:at + N]), plain)
        assert (out[:, :at] == 3).all() and (out[:, at + N:] == 3).all()
    pb.check(plain, *_want(c, GELU))
