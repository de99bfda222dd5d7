"""Gated feed-forward blocks of experts over sorted rows, and their gradients, against their definition in 64 bits."""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests import product_bounds as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _g(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _gauss(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=_g(seed), device=DEV) * scale).to(BF16)


def _off(counts, first=0):
    o = [first]
    for c in counts:
        o.append(o[-1] + c)
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def _case(counts, h, f, seed, extra=0, first=0):
    E, R = len(counts), first + sum(counts) + extra
    return {"x": _gauss((R, h), seed), "wgu": _gauss((E, 2 * f, h), seed + 1, h ** -0.5), "wd": _gauss((E, h, f), seed + 2, f ** -0.5),
            "dy": _gauss((R, h), seed + 3), "off": _off(counts, first), "counts": counts, "first": first}


def _spans(c):
    lo = c["first"]
    for e, n in enumerate(c["counts"]):
        yield e, lo, lo + n
        lo += n


def _check_forward(c, out):
    for e, lo, hi in _spans(c):
        if hi > lo:
            pb.check(out[lo:hi], *pb.ffn(c["x"][lo:hi].double(), c["wgu"][e].double(), c["wd"][e].double())[0], f"expert {e}")


def _check_backward(c, dx, dwgu, dwd):
    for e, lo, hi in _spans(c):
        if hi == lo:
            assert (dwgu[e] == 0).all() and (dwd[e] == 0).all()
            continue
        want = pb.ffn_grads(c["x"][lo:hi].double(), c["wgu"][e].double(), c["wd"][e].double(), c["dy"][lo:hi].double())
        for got, (v, err), name in zip((dx[lo:hi], dwgu[e], dwd[e]), want, ("dx", "dw_gate_up", "dw_down")):
            pb.check(got, v, err, f"{name} of expert {e}")


# rows of an expert: none, one, around 8, 16, 64 and 256; widths below and around tiles of 64, 128 and 256 and chunks of 64
COUNTS = [[1], [8], [9], [16], [17], [40], [256], [257], [300, 0, 5], [0, 0, 1, 0], [3, 1, 0, 2, 1, 1, 0, 5, 3], [70, 64, 63, 65, 0, 128, 1],
          [513, 15, 240, 272]]
SHAPES = [(8, 8), (64, 64), (72, 136), (264, 120), (520, 264), (1032, 344), (2056, 8), (8, 2056)]


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("h,f", SHAPES)
def test_block_and_its_gradients(h, f, counts):
    c = _case(counts, h, f, h + f)
    _check_forward(c, binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]))
    _check_backward(c, *binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"]))
    assert binding.operator_status() == binding.OK


@pytest.mark.parametrize("R", [1, 5, 16, 17, 33, 100, 250, 700])
def test_one_expert_without_offsets(R):
    c = _case([R], 1096, 392, R)
    _check_forward(c, binding.ffn(c["x"], c["wgu"], c["wd"]))
    _check_backward(c, *binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"]))


# one tile's contraction dealt along k (few tiles of long rows), and many tiles a pair
@pytest.mark.parametrize("counts,h,f", [([20], 7168, 2048), ([100, 30], 4096, 512), ([60] * 40, 264, 520), ([300] * 24, 520, 264),
                                        ([5] * 300, 136, 72), ([2] * 8, 2048, 1024), ([1] * 2048, 16, 16), ([0] * 2000 + [3] * 48, 64, 32)])
def test_every_way_to_deal_the_work(counts, h, f):
    c = _case(counts, h, f, len(counts))
    _check_forward(c, binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]))
    _check_backward(c, *binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"]))


@pytest.mark.parametrize("counts,extra,first", [([3, 2], 4, 0), ([70, 30, 1], 50, 0), ([300, 280], 400, 0), ([5, 4], 3, 2), ([90, 33], 20, 40)])
def test_rows_of_no_expert_are_left_alone_and_reach_nothing(counts, extra, first):
    """They hold NaN and infinities: no other row, and no gradient of a matrix, may see them."""
    h, f = 264, 136
    c = _case(counts, h, f, 5, extra, first)
    lo, hi = first, first + sum(counts)
    for name in ("x", "dy"):
        c[name][:lo], c[name][hi::2], c[name][hi + 1::2] = float("nan"), float("inf"), float("nan")
    out, dx = _gauss(c["x"].shape, 6), _gauss(c["x"].shape, 7)
    kept = out.clone(), dx.clone()
    binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"], out=out)
    got = binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"], dx=dx)
    _check_forward(c, out)
    _check_backward(c, *got)
    for a, b in zip((out, dx), kept):
        assert torch.equal(a[:lo], b[:lo]) and torch.equal(a[hi:], b[hi:])


@pytest.mark.parametrize("counts", [[3, 4, 5], [100, 30, 90]])
def test_values_that_are_not_finite_stay_with_their_row_and_expert(counts):
    h, f = 136, 72
    c = _case(counts, h, f, 8)
    clean, clean_b = binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]), binding.ffn_backward(
        c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])
    bad = counts[0] + 1                               # a row of expert 1
    c["x"][bad, 3] = float("nan")
    out, (dx, dwgu, dwd) = binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]), binding.ffn_backward(
        c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])
    rest = [r for r in range(sum(counts)) if r != bad]
    assert torch.isnan(out[bad]).all() and torch.equal(out[rest], clean[rest])
    assert torch.isnan(dx[bad]).all() and torch.equal(dx[rest], clean_b[0][rest])
    assert torch.isnan(dwgu[1]).all() and torch.isnan(dwd[1]).all()
    for e in (0, 2):
        assert torch.equal(dwgu[e], clean_b[1][e]) and torch.equal(dwd[e], clean_b[2][e])


def test_large_gates_saturate():
    """Gates far out: silu is 0 or the gate itself, nothing overflows on the way."""
    h, f, R = 64, 64, 40
    x = torch.full((R, h), 8.0, dtype=BF16, device=DEV)
    wgu = torch.zeros((1, 2 * f, h), dtype=BF16, device=DEV)
    wgu[0, :f // 2], wgu[0, f // 2:f], wgu[0, f:] = 4.0, -4.0, 0.25       # gates of +-2048, up 128
    wd = torch.zeros((1, h, f), dtype=BF16, device=DEV)
    wd[0, :, 0], wd[0, :, f - 1] = 1.0, 1.0
    for rows in (3, R):
        out = binding.ffn(x[:rows], wgu, wd)
        assert (out == 2048.0 * 128.0).all()
        dx, dwgu, dwd = binding.ffn_backward(x[:rows], wgu, wd, torch.ones_like(x[:rows]))
        assert all(torch.isfinite(t).all() for t in (dx, dwgu, dwd))
        assert (dwd[0, :, :f // 2] == 2048.0 * 128.0 * rows).all() and (dwd[0, :, f // 2:] == 0).all()


@pytest.mark.parametrize("counts", [[6, 5], [200, 90]])
def test_strides_are_followed(counts):
    h, f = 136, 200
    c = _case(counts, h, f, 9)
    wide = [_gauss((sum(counts), h + pad), 10 + pad) for pad in (8, 24, 16, 40)]
    x, dy, out, dx = (w[:, at:at + h] for w, at in zip(wide, (8, 16, 0, 32)))
    x.copy_(c["x"])
    dy.copy_(c["dy"])
    kept = [w.clone() for w in wide]
    binding.ffn(x, c["wgu"], c["wd"], expert_off=c["off"], out=out)
    got = binding.ffn_backward(x, c["wgu"], c["wd"], dy, expert_off=c["off"], dx=dx)
    _check_forward(c, out)
    _check_backward(c, *got)
    for w, k, at in zip(wide[2:], kept[2:], (0, 32)):
        assert torch.equal(w[:, :at], k[:, :at]) and torch.equal(w[:, at + h:], k[:, at + h:])


def test_equal_calls_give_equal_bits():
    c = _case([300, 7, 0, 90, 513], 520, 264, 11)
    first = [binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]),
             *binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])]
    for _ in range(5):
        again = [binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]),
                 *binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])]
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_gradients_against_differences():
    """Along a direction D of each input the loss <dout, out> changes by <gradient, D>.  The central difference of the definition in
    64 bits, steps of 2^-10, is off by less than 1e-5 of the sizes involved; the gradients by their bounds."""
    c = _case([13, 40], 72, 48, 12)
    leaves = [c["x"].double(), c["wgu"].double(), c["wd"].double()]

    def loss(x, wgu, wd):
        total = 0.0
        for e, lo, hi in _spans(c):
            z = x[lo:hi] @ wgu[e].T
            y = (torch.nn.functional.silu(z[:, :48]) * z[:, 48:]) @ wd[e].T
            total = total + (y * c["dy"][lo:hi].double()).sum()
        return total

    got = binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])
    bounds = [torch.zeros_like(v) for v in leaves]
    for e, lo, hi in _spans(c):
        w = pb.ffn_grads(c["x"][lo:hi].double(), c["wgu"][e].double(), c["wd"][e].double(), c["dy"][lo:hi].double())
        for b, at, (v, err) in zip(bounds, (slice(lo, hi), e, e), w):
            b[at] = err + pb.BF16_HALF * (v.abs() + err)
    for i, (g, b) in enumerate(zip(got, bounds)):
        D = torch.randn(leaves[i].shape, generator=_g(20 + i), device=DEV, dtype=torch.float64)
        D /= D.norm()
        step = 2.0 ** -10
        up, down = list(leaves), list(leaves)
        up[i], down[i] = leaves[i] + step * D, leaves[i] - step * D
        want = (loss(*up) - loss(*down)) / (2 * step)
        assert abs((g.double() * D).sum() - want) <= (b * D.abs()).sum() + 1e-5 * g.double().norm()


@pytest.mark.parametrize("off", [[0, 64, 0, 64], [0, 10, 9, 20], [64, 0, 0, 0], [0, 0, 70, 6]])
@pytest.mark.parametrize("R", [16, 64, 200])
def test_offsets_that_decrease_write_nothing(off, R):
    c = _case([R, 0, 0], 64, 40, 13)
    o = torch.tensor(off, dtype=torch.int32, device=DEV)
    out, dx = torch.full_like(c["x"], 5.0), torch.full_like(c["x"], 6.0)
    dwgu, dwd = torch.full_like(c["wgu"], 7.0), torch.full_like(c["wd"], 8.0)
    binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=o, out=out)
    binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=o, dx=dx, dw_gate_up=dwgu, dw_down=dwd)
    assert (out == 5).all() and (dx == 6).all() and (dwgu == 7).all() and (dwd == 8).all()


@pytest.mark.parametrize("R", [12, 60])
def test_offsets_beyond_the_rows_are_cut(R):
    c = _case([R // 2, R // 2], 64, 40, 14)
    want, want_b = binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=c["off"]), binding.ffn_backward(
        c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])
    o = torch.tensor([-5, R // 2, 10 ** 9], dtype=torch.int32, device=DEV)
    room, room_b = torch.full((R + 40, 64), 3.0, dtype=BF16, device=DEV), torch.full((R + 40, 64), 3.0, dtype=BF16, device=DEV)
    binding.ffn(c["x"], c["wgu"], c["wd"], expert_off=o, out=room[:R])
    got = binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=o, dx=room_b[:R])
    assert torch.equal(room[:R], want) and all(torch.equal(a, b) for a, b in zip(got, want_b))
    assert (room[R:] == 3).all() and (room_b[R:] == 3).all()


def test_no_rows():
    wgu, wd = _gauss((3, 32, 24), 1), _gauss((3, 24, 16), 2)
    x = torch.empty((0, 24), dtype=BF16, device=DEV)
    off = torch.zeros(4, dtype=torch.int32, device=DEV)
    assert binding.ffn(x, wgu, wd, expert_off=off).shape == (0, 24)
    dx, dwgu, dwd = binding.ffn_backward(x, wgu, wd, x, expert_off=off)
    assert dx.shape == (0, 24) and (dwgu == 0).all() and (dwd == 0).all()
    x = _gauss((40, 24), 3)                            # rows, but no expert has one
    out = torch.ones_like(x)
    binding.ffn(x, wgu, wd, expert_off=off, out=out)
    _, dwgu, dwd = binding.ffn_backward(x, wgu, wd, x, expert_off=off, dx=out)
    assert (out == 1).all() and (dwgu == 0).all() and (dwd == 0).all()


def test_captured_calls_follow_new_offsets_and_two_graphs_share_nothing():
    h, f, E, R = 264, 136, 6, 150

    def fill(seed):
        cut = sorted(torch.randint(0, R + 1, (E - 1,), generator=torch.Generator().manual_seed(seed)).tolist())
        return {"x": _gauss((R, h), seed), "dy": _gauss((R, h), seed + 50),
                "off": torch.tensor([0] + cut + [R], dtype=torch.int32, device=DEV)}

    wgu, wd = _gauss((E, 2 * f, h), 1, h ** -0.5), _gauss((E, h, f), 2, f ** -0.5)

    def step(s):
        small = binding.ffn(s["x"][:9], wgu[:1], wd[:1])
        return (binding.ffn(s["x"], wgu, wd, expert_off=s["off"]), small,
                *binding.ffn_backward(s["x"], wgu, wd, s["dy"], expert_off=s["off"]))

    states, graphs, outs = [fill(1), fill(2)], [], []
    for s in states:
        step(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    for i, s in enumerate(states):
        for n, t in fill(5 + i).items():
            s[n].copy_(t)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s, got in zip(states, outs):
        assert all(torch.equal(a, b) for a, b in zip(got, step(s)))
    assert binding.operator_status() == binding.OK


def test_results_are_there_for_what_comes_next_in_the_stream():
    """The backward call's last kernels start early; what follows it in the stream must still see all of its outputs."""
    c = _case([40, 3, 90], 520, 264, 15)
    want = [t.clone() for t in binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"])]
    outs = [torch.empty_like(t) for t in want]
    sums = []
    for _ in range(50):
        for t in outs:
            t.fill_(9.0)
        binding.ffn_backward(c["x"], c["wgu"], c["wd"], c["dy"], expert_off=c["off"], dx=outs[0], dw_gate_up=outs[1], dw_down=outs[2])
        sums.append([(a != b).sum() for a, b in zip(outs, want)])
    assert all(int(n) == 0 for s in sums for n in s)


def test_rows_beyond_32_bit_offsets():
    """More than 2^31 values of x: the last expert's rows against their definition."""
    h, f, tail = 4096, 16, 70
    R = 2 ** 31 // h + 300
    x, out = torch.zeros((R, h), dtype=BF16, device=DEV), torch.zeros((R, h), dtype=BF16, device=DEV)
    x[-tail:] = _gauss((tail, h), 1)
    wgu, wd = _gauss((2, 2 * f, h), 2, h ** -0.5), _gauss((2, h, f), 3, f ** -0.5)
    off = torch.tensor([0, R - tail, R], dtype=torch.int32, device=DEV)
    binding.ffn(x, wgu, wd, expert_off=off, out=out)
    pb.check(out[-tail:], *pb.ffn(x[-tail:].double(), wgu[1].double(), wd[1].double())[0])
    dy = torch.zeros_like(x)
    dy[-tail:] = _gauss((tail, h), 4)
    dx, dwgu, dwd = binding.ffn_backward(x, wgu, wd, dy, expert_off=off, dx=out)
    for got, (v, e) in zip((dx[-tail:], dwgu[1], dwd[1]), pb.ffn_grads(x[-tail:].double(), wgu[1].double(), wd[1].double(), dy[-tail:].double())):
        pb.check(got, v, e)
    assert (dwgu[0] == 0).all() and (dwd[0] == 0).all()


def test_wrapper_refuses_what_does_not_fit():
    x, wgu, wd = _gauss((6, 32), 1), _gauss((2, 48, 32), 2), _gauss((2, 32, 24), 3)
    off = torch.tensor([0, 2, 6], dtype=torch.int32, device=DEV)
    q, b = binding.ffn, binding.ffn_backward
    bad = [lambda: q(x, wgu, wd), lambda: q(x.float(), wgu, wd, expert_off=off), lambda: q(x, wgu.float(), wd, expert_off=off),
           lambda: q(x, wgu, wd, expert_off=off[:2]), lambda: q(x, wgu, wd, expert_off=off.long()), lambda: q(x, wgu[:, :40], wd, expert_off=off),
           lambda: q(x, wgu, wd.transpose(1, 2), expert_off=off), lambda: q(x[:, :24], wgu, wd, expert_off=off),
           lambda: q(x.cpu(), wgu, wd, expert_off=off), lambda: q(x, wgu, wd, expert_off=off, out=x),
           lambda: q(x, wgu, wd, expert_off=off, out=x[:4]), lambda: q(_gauss((6, 33), 1)[:, 1:], wgu, wd, expert_off=off),
           lambda: q(x[:, :28].contiguous(), wgu[:, :, :28].contiguous(), wd[:, :28].contiguous(), expert_off=off),
           lambda: b(x, wgu, wd, x[:5], expert_off=off), lambda: b(x, wgu, wd, x, expert_off=off, dx=x),
           lambda: b(x, wgu, wd, x, expert_off=off, dw_down=wd), lambda: b(x, wgu, wd, x.float(), expert_off=off),
           lambda: b(x, wgu, wd, x, expert_off=off, dw_gate_up=wgu[:1])]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()
