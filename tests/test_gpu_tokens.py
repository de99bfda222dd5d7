"""Tokens sorted by expert and back (sort_pairs, dispatch, combine and their gradients) against plain definitions."""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests.bounds import Bounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _routing(T, k, n, seed, drop=0.0, distinct=True):
    g = _gen(seed)
    if distinct:
        idx = torch.rand((T, n), generator=g, device=DEV).topk(k, dim=1).indices.to(torch.int32)
    else:
        idx = torch.randint(0, n, (T, k), generator=g, device=DEV, dtype=torch.int32)
    if drop:
        gone = torch.rand((T, k), generator=g, device=DEV) < drop
        other = torch.randint(0, 4, (T, k), generator=g, device=DEV)
        bad = torch.tensor([-1, n, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=DEV)[other]
        idx = torch.where(gone, bad, idx)
    return idx, torch.rand((T, k), generator=g, device=DEV)


def _want_sort(idx, n):
    flat = idx.reshape(-1).cpu().tolist()
    lists = {e: [] for e in range(n)}
    for p, e in enumerate(flat):
        if 0 <= e < n:
            lists[e].append(p)
    off, rows = [0], []
    for e in range(n):
        rows += lists[e]
        off.append(len(rows))
    pair = [-1] * len(flat)
    for r, p in enumerate(rows):
        pair[p] = r
    return off, pair, rows + [-1] * (len(flat) - len(rows))


def _check_sort(idx, n):
    off, pair_row, row_pair = binding.sort_pairs(idx, n)
    w_off, w_pair, w_row = _want_sort(idx, n)
    assert off.tolist() == w_off
    assert pair_row.reshape(-1).tolist() == w_pair
    assert row_pair.tolist() == w_row
    return off, pair_row, row_pair


# around the sizes at which the form changes: 32 pairs a warp step, 1536 pairs in one block, 1024 pairs a block beyond;
# experts around the counters' limits (512 experts x 32 warps, 2048 experts x 8 warps)
@pytest.mark.parametrize("T,k,n", [(0, 4, 8), (1, 1, 1), (1, 8, 256), (16, 8, 256), (33, 1, 7), (31, 3, 33), (512, 8, 256),
                                   (410, 10, 864), (409, 10, 2048), (128, 32, 2047), (513, 8, 256), (4097, 1, 2048),
                                   (2048, 2, 5), (192, 8, 256), (193, 8, 256), (150, 10, 2048), (512, 2, 900), (1025, 1, 3), (4096, 8, 256), (1021, 10, 672), (3001, 7, 1), (20000, 8, 100)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_sort_is_stable_and_complete(T, k, n, drop):
    idx, _ = _routing(T, min(k, n) if n >= k else k, n, T + k + n, drop, distinct=n >= k)
    _check_sort(idx, n)


@pytest.mark.parametrize("T", [5, 3000])
def test_sort_extremes(T):
    k, n = 6, 64
    _check_sort(torch.full((T, k), 63, dtype=torch.int32, device=DEV), n)      # one expert takes all, repeatedly
    _check_sort(torch.full((T, k), -1, dtype=torch.int32, device=DEV), n)      # nothing is kept
    _check_sort(torch.zeros((T, k), dtype=torch.int32, device=DEV), 1)
    idx, _ = _routing(T, k, n, 3)
    idx[::2] = -1                                                              # padded tokens
    _check_sort(idx, n)


def _matrix(rows, cols, dtype, seed, layout):
    """A [rows, cols] matrix: dense, a column range of a wider one (16-byte aligned or not)."""
    g = _gen(seed)
    if layout == "dense":
        return torch.randn((rows, cols), generator=g, device=DEV).to(dtype)
    pad, at = (16, 8) if layout == "strided" else (7, 3)
    return torch.randn((rows, cols + pad), generator=g, device=DEV).to(dtype)[:, at:at + cols]


SHAPES = [(1, 1, 1, 1), (1, 8, 256, 7168), (3, 2, 5, 8), (16, 8, 256, 4096), (7, 32, 40, 72), (64, 10, 672, 1027),
          (129, 9, 16, 640), (1000, 3, 11, 33), (257, 8, 64, 2056)]


@pytest.mark.parametrize("layout", ["dense", "strided", "odd"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,k,n,h", SHAPES)
def test_rows_go_out_and_come_back(T, k, n, h, dtype, layout):
    """dispatch and dispatch_backward, combine and combine_backward, with dropped pairs: values, untouched rows."""
    idx, w = _routing(T, k, n, T + h, drop=0.2, distinct=n >= k)
    off, pair_row, row_pair = binding.sort_pairs(idx, n)
    R = T * k
    filled = int(off[-1])
    pairs = row_pair[:filled].long()
    x = _matrix(T, h, dtype, 1, layout)
    rows = _matrix(R + 3, h, dtype, 2, layout)
    kept = rows.clone()
    binding.dispatch(x, pair_row, rows=rows)
    assert torch.equal(rows[:filled], x[pairs // k]) and torch.equal(rows[filled:], kept[filled:])

    y = _matrix(R, h, dtype, 3, layout)
    y[filled:] = float("nan")                                  # behind the last row: must not be looked at
    out = _matrix(T, h, dtype, 4, layout)
    w = torch.where(pair_row < 0, torch.full_like(w, float("nan")), w)   # nor dropped pairs' weights
    binding.combine(y, pair_row, w, out=out)
    ok = (pair_row >= 0)
    take = torch.where(ok[:, :, None], y[pair_row.long().clamp(min=0)].double(), torch.zeros((), dtype=torch.float64, device=DEV))
    w64 = torch.where(ok, w, torch.zeros_like(w))
    (Bounded(take) * Bounded(w64[:, :, None])).sum(1).within(out, "out")

    dx = binding.dispatch_backward(y, pair_row, dx=_matrix(T, h, dtype, 5, layout))
    Bounded(take).sum(1).within(dx, "dx")

    dout = _matrix(T, h, dtype, 6, layout)
    drows = _matrix(R + 2, h, dtype, 7, layout)
    kept = drows.clone()
    big = _matrix(R + 2, h, dtype, 8, layout)
    _, dw = binding.combine_backward(dout, big, pair_row, w, drows=drows)
    assert torch.equal(drows[filled:], kept[filled:])
    (Bounded(dout[pairs // k]) * Bounded(w.reshape(-1)[pairs][:, None])).within(drows[:filled], "drows")
    got = (Bounded(dout.double()[:, None, :].expand(T, k, h)) *
           Bounded(torch.where(ok[:, :, None], big[pair_row.long().clamp(min=0)].double(),
                               torch.zeros((), dtype=torch.float64, device=DEV)))).sum(2)
    got.within(dw, "dw")
    assert (dw[~ok] == 0).all()


def test_gradients_are_the_adjoints_of_the_forward_calls():
    """<dispatch(x), d> = <x, dispatch_backward(d)>, and the derivative of <combine(y; w), d> along (v, s) by differences
    (combine is bilinear: the central difference in fp64 of its definition has no truncation error)."""
    T, k, n, h = 37, 5, 12, 129
    idx, w = _routing(T, k, n, 1, drop=0.2)
    off, pair_row, row_pair = binding.sort_pairs(idx, n)
    f = int(off[-1])
    x, d = _matrix(T, h, torch.float32, 1, "dense"), _matrix(T * k, h, torch.float32, 2, "dense")
    rows = binding.dispatch(x, pair_row)
    dx = binding.dispatch_backward(d, pair_row)
    left, right = (rows[:f].double() * d[:f].double()).sum(), (x.double() * dx.double()).sum()
    assert abs(left - right) <= (k + 2) * 2.0 ** -24 * (x.double().abs() * d.double().abs()[pair_row.long().clamp(min=0)].sum(1)).sum()

    y, dout = _matrix(T * k, h, torch.float32, 3, "dense"), _matrix(T, h, torch.float32, 4, "dense")
    v, s = _matrix(T * k, h, torch.float32, 5, "dense").double(), torch.randn((T, k), generator=_gen(6), device=DEV).double()
    drows, dw = binding.combine_backward(dout, y, pair_row, w)
    ok = (pair_row >= 0)[:, :, None]

    def loss(step):
        take = (y.double() + step * v)[pair_row.long().clamp(min=0)] * ok
        return (((w.double() + step * s)[:, :, None] * take).sum(1) * dout.double()).sum()

    difference = (loss(0.5) - loss(-0.5)) / 1.0
    along = (drows[:f].double() * v[:f]).sum() + (dw.double() * s).sum()
    size = (drows[:f].double().abs() * v[:f].abs()).sum() + (dout.double().abs()[:, None, :] * y.double().abs()[pair_row.long().clamp(min=0)] * s.abs()[:, :, None]).sum()
    assert abs(difference - along) <= (h + 2) * 2.0 ** -24 * size


def test_one_of_the_two_gradients_alone():
    T, k, n, h = 9, 4, 8, 256
    idx, w = _routing(T, k, n, 1)
    _, pair_row, _ = binding.sort_pairs(idx, n)
    y, dout = _matrix(T * k, h, torch.bfloat16, 3, "dense"), _matrix(T, h, torch.bfloat16, 4, "dense")
    drows, dw = binding.combine_backward(dout, y, pair_row, w)
    L, p = binding.lib(), binding._dptr
    only, alone = torch.zeros_like(drows), torch.zeros_like(dw)
    args = (T, k, h)
    assert L.deamoe_combine_backward(binding._stream(), 1, p(dout), h, None, 0, T * k, p(pair_row), p(w), *args, p(only), h, None) == 0
    assert L.deamoe_combine_backward(binding._stream(), 1, p(dout), h, p(y), h, T * k, p(pair_row), p(w), *args, None, 0, p(alone)) == 0
    assert torch.equal(only, drows) and torch.equal(alone, dw)


def test_row_indices_out_of_range_are_skipped():
    T, k, h = 4, 3, 64
    pair_row = torch.tensor([[0, 1, 2], [3, 100, 4], [-7, 5, 6], [2 ** 31 - 1, -2 ** 31, 7]], dtype=torch.int32, device=DEV)
    x = _matrix(T, h, torch.float32, 1, "dense")
    rows = torch.full((8, h), 9.0, device=DEV)
    binding.dispatch(x, pair_row, rows=rows)
    want = torch.stack([x[0], x[0], x[0], x[1], x[1], x[2], x[2], x[3]])
    assert torch.equal(rows, want)
    w = torch.ones((T, k), device=DEV)
    out = binding.combine(rows, pair_row, w)
    assert torch.equal(out, torch.stack([rows[0] + rows[1] + rows[2], rows[3] + rows[4], rows[5] + rows[6], rows[7]]))


def test_captured_steps_follow_new_routing_and_two_graphs_do_not_disturb_each_other():
    T, k, n, h = 700, 8, 64, 512                      # the sort's three-kernel form: it has a workspace

    def step(s):
        off, pair_row, row_pair = binding.sort_pairs(s["idx"], n)
        rows = binding.dispatch(s["x"], pair_row)
        return off, pair_row, row_pair, rows, binding.combine(rows, pair_row, s["w"])

    states, graphs, outs = [], [], []
    for i in range(2):
        idx, w = _routing(T, k, n, i)
        s = {"idx": idx, "w": w, "x": _matrix(T, h, torch.bfloat16, 10 + i, "dense")}
        step(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        states.append(s)
        graphs.append(g)
    for i, s in enumerate(states):                    # new data in the same buffers
        idx, w = _routing(T, k, n, 20 + i, drop=0.1)
        s["idx"].copy_(idx)
        s["w"].copy_(w)
        s["x"].copy_(_matrix(T, h, torch.bfloat16, 30 + i, "dense"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s, got in zip(states, outs):
        want = step(s)
        f = int(want[0][-1])
        for a, b in zip(got[:3], want[:3]):
            assert torch.equal(a, b)
        assert torch.equal(got[3][:f], want[3][:f]) and torch.equal(got[4], want[4])


def test_wrapper_refuses_what_does_not_fit():
    idx, w = _routing(4, 2, 8, 1)
    _, pair_row, _ = binding.sort_pairs(idx, 8)
    x = _matrix(4, 64, torch.bfloat16, 1, "dense")
    bad = [lambda: binding.sort_pairs(idx.long(), 8), lambda: binding.sort_pairs(idx, 0), lambda: binding.sort_pairs(idx, 4096),
           lambda: binding.sort_pairs(idx.cpu(), 8), lambda: binding.dispatch(x.half(), pair_row),
           lambda: binding.dispatch(x, pair_row.long()), lambda: binding.dispatch(x[:3], pair_row),
           lambda: binding.dispatch(x.t(), pair_row), lambda: binding.dispatch(x, pair_row, rows=x.float()),
           lambda: binding.combine(x, pair_row, w.double()), lambda: binding.combine(x, pair_row, w[:, :1]),
           lambda: binding.combine_backward(x, x.float(), pair_row, w),
           lambda: binding.dispatch(x[:, :1].expand(4, 64), pair_row), lambda: binding.combine(x, pair_row.reshape(-1), w),
           lambda: binding.dispatch(x, pair_row.reshape(-1)), lambda: binding.combine_backward(x, x[0], pair_row, w)]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()


def test_rows_beyond_32_bit_offsets():
    """Over 2^31 values of rows: the last tokens' rows out, back, and in the gradients."""
    T, k, n, h = 40000, 8, 64, 7168
    idx, w = _routing(T, k, n, 1)
    _, pair_row, row_pair = binding.sort_pairs(idx, n)
    assert T * k * h > 2 ** 31
    x = torch.randn((T, h), generator=_gen(2), device=DEV).to(torch.bfloat16)
    rows = binding.dispatch(x, pair_row)
    tail = slice(T * k - 100, T * k)
    assert torch.equal(rows[tail], x[row_pair[tail].long() // k])
    last = pair_row[-50:].long()
    ones = torch.ones_like(w)
    Bounded(x[-50:, None].double().expand(50, k, h)).sum(1).within(binding.combine(rows, pair_row, ones)[-50:], "out")
    drows, dw = binding.combine_backward(x, rows, pair_row, w)
    (Bounded(x[row_pair[tail].long() // k]) * Bounded(w.reshape(-1)[row_pair[tail].long()][:, None])).within(drows[tail], "drows")
    (Bounded(x[-50:, None].double().expand(50, k, h)) * Bounded(rows[last].double())).sum(2).within(dw[-50:], "dw")
