"""Sums of many terms of one sign, where a sum that is cut at every step loses most: weight gradients over tens of thousands to millions
of rows, and products of very wide rows.

The tensor cores' fp32 sums lose some 6e-9 of a same-signed sum a term, so a stretch of 32768 terms loses 2e-4 of it; the
stretches are added with one rounding each.  LOSS is that with a quarter to spare; half a step of bf16 is 2e-3 to 4e-3.
"""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests import product_bounds as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
LOSS = 2.5e-4


def _positive(shape, seed, scaled=None):
    """Values around one; scaled: with a factor a row (0) or a column (1), so that sums do not all round alike."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.rand(shape, generator=g, device=DEV) + 0.5
    if scaled is not None:
        v *= 1 + torch.rand([n if i == scaled else 1 for i, n in enumerate(shape)], generator=g, device=DEV)
    return v.to(BF16)


def _over_rows(a, b):
    """a^T b in 64 bits, some rows at a time."""
    v = torch.zeros((a.shape[1], b.shape[1]), dtype=torch.float64, device=DEV)
    for i in range(0, a.shape[0], 1 << 17):
        v += a[i:i + (1 << 17)].double().T @ b[i:i + (1 << 17)].double()
    return v


def _check_sums(got, v, terms, what="", distinct=None):
    """Half a step of bf16 at the value itself, the loss of a stretch, and a rounding a stretch.  distinct: how many of the values are
    not others times a power of two (and so round by themselves)."""
    e = (LOSS + (terms // 32768 + 1) * 2.0 ** -24) * v.abs()
    half = torch.exp2(torch.floor(torch.log2(v.abs() + e)) - 8)
    worst = ((got.double() - v).abs() / (half + e)).max().item()
    assert worst <= 1, (what, worst)
    bias = ((got.double() - v) / v).mean().item()
    # roundings are independent of one another: their mean over n values is within 5 of 2^-8 / sqrt(3 n)
    assert abs(bias) <= LOSS + 5 * 2.0 ** -8 / (3 * (distinct or v.numel())) ** 0.5, (what, bias)


@pytest.mark.parametrize("T,K,N", [(32768, 264, 136), (32769, 136, 264), (65536, 520, 64), (131072 + 77, 264, 136), ((1 << 20) + 64, 72, 136),
                                   ((1 << 22) + 4381, 64, 72)])
def test_weight_gradient_of_many_tokens(T, K, N):
    x, d, w = _positive((T, K), 1, 1), _positive((T, N), 2, 1), _positive((N, K), 3)
    dx, dw, db = binding.product_backward(x, w, d, bias=torch.zeros(N, device=DEV))
    _check_sums(dw, _over_rows(d, x), T, "dweight")
    for rows in (slice(0, 40), slice(T - 40, T)):
        pb.check(dx[rows], *pb.dot(d[rows].double(), None, w.double().T, None))
    assert binding.operator_status() == binding.OK


@pytest.mark.parametrize("counts", [[40000], [70001, 0, 32768, 5, 100000], [32832, 3, 65537], [1 << 20, 12, 1 << 19]])
def test_experts_of_many_rows(counts):
    """Gates of 64 (SiLU is the gate itself) and ups of 4 from a column of x that is 16, a down matrix that hands feature i's gradient to it
    from column i: every operand of the weight gradients is exact, and so is what they are sums of."""
    h, f, E, R = 136, 72, len(counts), sum(counts)
    x, dy = _positive((R, h), 1, 1), _positive((R, h), 2, 1)
    x[:, 0] = 16.0
    wgu, wd = torch.zeros((E, 2 * f, h), dtype=BF16, device=DEV), torch.zeros((E, h, f), dtype=BF16, device=DEV)
    wgu[:, :f, 0], wgu[:, f:, 0] = 4.0, 0.25
    wd[:, torch.arange(f), torch.arange(f)] = 1.0
    off = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
    dx, dwgu, dwd = binding.ffn_backward(x, wgu, wd, dy, expert_off=off)
    assert binding.operator_status() == binding.OK
    lo = 0
    for e, n in enumerate(counts):
        hi = lo + n
        if n == 0:
            assert (dwgu[e] == 0).all() and (dwd[e] == 0).all()
            continue
        each = _over_rows(dy[lo:hi, :f], x[lo:hi])
        _check_sums(dwgu[e], torch.cat([4 * each, 64 * each]), n, f"dw_gate_up of expert {e}", each.numel())
        _check_sums(dwd[e], (256 * dy[lo:hi].double().sum(0))[:, None].expand(h, f), n, f"dw_down of expert {e}", h)
        lo = hi


def _wide(T, K, N, kind):
    x, w = _positive((T, K), 1, 0), _positive((N, K), 2, 0)
    if kind == "bf16":
        return x, w, {}
    return (x.float() * 64).to(F8), (w.float() * 64).to(F8), {"x_scale": torch.full((T,), 2.0 ** -6, device=DEV),
                                                             "weight_scale": torch.full((N,), 2.0 ** -6, device=DEV)}


# more than a stretch: whole contractions of many tiles, and parts of few
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(2560, 66000, 4096), (2500, 131104, 4100), (40, 1 << 20, 72), (300, 1 << 20, 33)])
def test_product_of_wide_rows(T, K, N, kind):
    K = K // 16 * 16
    x, w, scales = _wide(T, K, N, kind)
    y = binding.product(x, w, **scales)
    v = _over_rows(x.float().T, w.float().T) if kind == "bf16" else _over_rows(x.float().T, w.float().T) * 2.0 ** -12
    _check_sums(y, v, K)
    assert binding.operator_status() == binding.OK


@pytest.fixture
def tight(monkeypatch):
    """The bounds' sum of products, with the loss of a stretch for its additions."""
    def dot(a, ea, b, eb):
        n = a.shape[1]
        size = (a.abs() + (0 if ea is None else ea)) @ (b.abs() + (0 if eb is None else eb)).T
        e = (LOSS + (n // 32768 + 9) * 2.0 ** -23) * size
        if ea is not None:
            e = e + ea @ b.abs().T
        if eb is not None:
            e = e + (a.abs() + (0 if ea is None else ea)) @ eb.T
        return a @ b.T, e
    monkeypatch.setattr(pb, "dot", dot)


@pytest.mark.parametrize("act", [binding.SIGMA_SILU, binding.SIGMA_GELU])
@pytest.mark.parametrize("T,K,N", [(300, 40008, 264), (90, 264, 40008), (64, 70000, 72)])
def test_epilogues_behind_wide_rows(tight, T, K, N, act):
    x, w, d, bias = _positive((T, K), 1, 0), _positive((N, K), 2, 0), _positive((T, N), 3), -_positive((N,), 4)
    w *= 1.0 / K                                       # z of one to four before the bias
    r = _positive((T, N), 5)
    y = binding.product(x, w, bias=bias, act=act, residual=r)
    z, e = pb.dot(x.double(), None, w.double(), None)
    z, e = pb.plus(z, e, bias.double()[None, :], torch.zeros_like(z))
    a, ea = pb.act(act, z, e)
    pb.check(y, *pb.plus(a, ea, r.double(), torch.zeros_like(a)))
    dx, dw, db = binding.product_backward(x, w, d, bias=bias, act=act)
    dz, eb = pb.times(d.double(), torch.zeros_like(z), *pb.act_grad(act, z, e))
    pb.check(db, dz.sum(0), eb.sum(0) + (T + 8) * 2.0 ** -24 * (dz.abs() + eb).sum(0), "dbias")
    dz, e = pb.to_bf16(dz, eb)
    pb.check(dx, *pb.dot(dz, e, w.double().T, None), "dx")
    pb.check(dw, *pb.dot(dz.T, e.T, x.double().T, None), "dweight")
    assert binding.operator_status() == binding.OK


@pytest.mark.parametrize("counts,h,f", [([40, 300], 40008, 136), ([40, 300], 136, 40008), ([20], 1 << 20, 8), ([33], 8, 1 << 20)])
def test_blocks_of_wide_rows(tight, counts, h, f):
    E, R = len(counts), sum(counts)
    x, dy = _positive((R, h), 1, 0), _positive((R, h), 2)
    wgu, wd = _positive((E, 2 * f, h), 3), _positive((E, h, f), 4)
    wgu *= 1.0 / h
    off = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
    out = binding.ffn(x, wgu, wd, expert_off=off)
    got = binding.ffn_backward(x, wgu, wd, dy, expert_off=off)
    lo = 0
    for e, n in enumerate(counts):
        rows = slice(lo, lo + n)
        lo += n
        args = [t.double() for t in (x[rows], wgu[e], wd[e])]
        pb.check(out[rows], *pb.ffn(*args)[0], f"expert {e}")
        want = pb.ffn_grads(*args, dy[rows].double())
        for g, (v, err), name in zip((got[0][rows], got[1][e], got[2][e]), want, ("dx", "dw_gate_up", "dw_down")):
            pb.check(g, v, err, f"{name} of expert {e}")
    assert binding.operator_status() == binding.OK


def test_equal_calls_give_equal_bits_and_graphs_share_no_sums():
    T, K, N = 100001, 264, 72
    w, bias = _positive((N, K), 1), torch.zeros(N, device=DEV)

    def step(s):
        return binding.product_backward(s["x"], w, s["d"], bias=bias)

    states = [{"x": _positive((T, K), i, 1), "d": _positive((T, N), i + 5, 1)} for i in (2, 3)]
    want = [[t.clone() for t in step(s)] for s in states]
    assert all(torch.equal(a, b) for s, ws in zip(states, want) for a, b in zip(step(s), ws))
    graphs, outs = [], []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, ws in zip(outs, want) for a, b in zip(o, ws))


def test_contraction_that_takes_longer_than_a_wait():
    """800 million rows in one tile: 12.6 million chunks at 0.3 us, longer than the 2 s after which a wait gives up where nothing moves.  Zeros but for
    a row for each output, at the ends, at edges of stretches and in the last, ragged chunk."""
    T, K, N = 3 * (1 << 28) + 77, 8, 8
    x, d, w = torch.ones((T, K), dtype=BF16, device=DEV), torch.zeros((T, N), dtype=BF16, device=DEV), torch.zeros((N, K), dtype=BF16, device=DEV)
    at = [0, 32767, 32768, 1 << 28, (1 << 29) - 1, 1 << 29, T - 14, T - 1]
    for i, t in enumerate(at):
        d[t, i] = float(1 << i)
        x[t] = 1.0 + i / 8
    dx, dw, _ = binding.product_backward(x, w, d)
    assert binding.operator_status() == binding.OK
    del dx
    assert torch.equal(dw.double(), _over_rows(d[at], x[at]))


EDGES = ([0, 7, 8, 15, 16, 62, 63, 64], [65, 127, 128, 255, 256, 511, 512, 32767], [32768, 65535, 65536, 65599, 131071, 131072, 262143, 262144],
         [-1, -13, -14, -77, -78, -141, -142, 1 << 21])


@pytest.mark.parametrize("at", EDGES)
def test_every_row_of_millions_counts_once(at):
    """Sums that are exact: a row for each output at the edges of blocks, chunks and stretches, zeros elsewhere; and ones everywhere, whose
    sum in fp32 is the number of rows."""
    T, K, N = 65536 * 64 + 77, 8, 8
    x, d, w = torch.ones((T, K), dtype=BF16, device=DEV), torch.zeros((T, N), dtype=BF16, device=DEV), torch.zeros((N, K), dtype=BF16, device=DEV)
    for i, t in enumerate(at):
        d[t, i], x[t] = float(1 << i), 1.0 + i / 8
    dx, dw, db = binding.product_backward(x, w, d, bias=torch.zeros(N, device=DEV))
    assert torch.equal(dw.double(), _over_rows(d[at], x[at])) and torch.equal(db.double(), d[at].double().sum(0)) and (dx == 0).all()
    db = binding.product_backward(x, w, torch.ones_like(d), bias=torch.zeros(N, device=DEV))[2]
    assert (db == float(T)).all()
    # the derivative of SiLU at 0 is a half: the same sums behind an activation
    dw, db = binding.product_backward(x, w, d, bias=torch.zeros(N, device=DEV), act=binding.SIGMA_SILU)[1:]
    assert torch.equal(2 * dw.double(), _over_rows(d[at], x[at])) and torch.equal(2 * db.double(), d[at].double().sum(0))
    assert binding.operator_status() == binding.OK


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(16, 1 << 20, 256), (5, 1 << 20, 1000), (16, 400016, 4096), (8, 140000, 8192), (3, 262144 + 16, 7200)])
def test_few_rows_of_great_width(T, K, N, kind):
    x, w, scales = _wide(T, K, N, kind)
    y = binding.product(x, w, **scales)
    v = _over_rows(x.float().T, w.float().T) * (1.0 if kind == "bf16" else 2.0 ** -12)
    _check_sums(y, v, K)


@pytest.mark.parametrize("R,h,f", [(9, 1 << 20, 24), (16, 72, 1 << 20), (4, 300008, 3600)])
def test_a_block_of_few_rows_of_great_width(tight, R, h, f):
    x, wgu, wd = _positive((R, h), 1, 0), _positive((1, 2 * f, h), 3), _positive((1, h, f), 4)
    wgu *= 1.0 / h
    out = binding.ffn(x, wgu, wd)
    for lo in range(0, h, 1 << 16):                    # columns of the output some at a time, for their room in 64 bits
        hi = min(h, lo + (1 << 16))
        if lo == 0:
            _, (g, eg, u, eu, hh, eh) = pb.ffn(x.double(), wgu[0].double(), wd[0, :8].double())
        pb.check(out[:, lo:hi], *pb.dot(hh, eh, wd[0, lo:hi].double(), None))
