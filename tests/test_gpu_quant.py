"""Products with 4-bit matrices against the definition in 64 bits."""
import pytest
import torch

from paper_2608_14385_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def _matrices(E, N, K, group, zeros, sdtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    G = -(-K // group)
    codes = torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = ((torch.rand((E, N, G), generator=g, device=DEV) - 0.3) * 0.02).to(sdtype)
    z = torch.randint(0, 16, (E, N, G), generator=g, device=DEV, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def _widened(codes, scales, z, group, K):
    low, high = (codes & 15).double(), (codes >> 4).double()
    q = torch.stack([low, high], dim=-1).flatten(-2)
    col = torch.arange(K, device=DEV) // group
    return (q - (8.0 if z is None else z.double()[..., col])) * scales.double()[..., col]


def _want(codes, scales, z, group, x, experts, sources, swiglu):
    """The products of every row in 64 bits, and what fp32 may be off by before the output's rounding: a sum of K + 2 G
    terms, each addition good to one unit (2^-23: the tensor cores cut rather than round), fp32 x carried to 2^-23."""
    K = x.shape[1]
    N = codes.shape[1]
    got = torch.zeros((len(experts), N), dtype=torch.float64, device=DEV)
    err = torch.zeros_like(got)
    for e in sorted(set(experts)):
        rows = [r for r in range(len(experts)) if experts[r] == e]
        w = _widened(codes[e], scales[e], None if z is None else z[e], group, K)
        src = [sources[r] for r in rows]
        xs = torch.stack([x[s].double() if 0 <= s < x.shape[0] else torch.zeros(K, dtype=torch.float64, device=DEV) for s in src])
        got[rows] = xs @ w.T
        err[rows] = (K + 2 * scales.shape[2] + 8) * 2.0 ** -23 * (xs.abs() @ w.abs().T)
    if swiglu:
        F = N // 2
        v, u, ev, eu = got[:, :F], got[:, F:], err[:, :F], err[:, F:]
        silu = v * torch.sigmoid(v)
        es = 1.1 * ev + 8 * 2.0 ** -24 * (silu.abs() + 1.1 * ev)
        got, err = silu * u, (silu.abs() + es) * eu + es * u.abs() + 2.0 ** -24 * (silu * u).abs()
    return got, err


def _check(got, want, err):
    half = torch.finfo(got.dtype).eps / 2
    bound = err + half * (want.abs() + err) + torch.finfo(got.dtype).tiny
    diff = (got.double() - want).abs()
    assert (diff <= bound).all(), (diff / bound).max().item()


def _routed(T, k, E, seed, skew=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    score = torch.rand((T, E), generator=g, device=DEV)
    if skew:
        score[:, :2] += 0.8
    idx = score.topk(k, dim=1).indices.to(torch.int32)
    off, _, row_pair = binding.sort_pairs(idx, E)
    o = off.tolist()
    experts = [e for e in range(E) for _ in range(o[e], o[e + 1])]
    return off, row_pair, experts, [p // k for p in row_pair.tolist()]


# one and several rows, around 8-row passes; widths around 16-row tiles; columns around 256-column steps and short groups
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,zeros,sdtype", [(32, True, BF16), (64, False, F32), (128, True, F32), (128, False, BF16)])
@pytest.mark.parametrize("T,N,K", [(1, 1, 32), (1, 16, 128), (1, 4096, 7168), (2, 17, 96), (3, 100, 1056), (7, 33, 160),
                                   (8, 48, 224), (9, 1003, 2048), (20, 66, 608), (33, 130, 1408), (70, 24, 384), (2, 40, 9248)])
def test_one_matrix(T, N, K, group, zeros, sdtype, dtype):
    codes, scales, z = _matrices(1, N, K, group, zeros, sdtype, T + N)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(K), device=DEV).to(dtype)
    got = binding.quant_product(codes, scales, x, group, zeros=z)
    _check(got, *_want(codes, scales, z, group, x, [0] * T, list(range(T)), False))
    if N % 2 == 0:
        got = binding.quant_product(codes, scales, x, group, zeros=z, swiglu=True)
        _check(got, *_want(codes, scales, z, group, x, [0] * T, list(range(T)), True))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,k,E,N,K,group,zeros,skew", [
    (1, 8, 32, 128, 512, 128, False, False), (4, 2, 16, 96, 1408, 64, True, False), (37, 2, 16, 1003, 1056, 32, True, False),
    (16, 8, 64, 64, 768, 128, False, False), (50, 3, 5, 40, 320, 64, True, True), (128, 2, 4, 34, 256, 128, False, True),
    (3, 1, 300, 32, 128, 32, False, False), (2, 2, 2, 18, 64, 64, True, False), (60, 4, 2048, 16, 96, 32, True, False)])
def test_experts_over_sorted_rows(T, k, E, N, K, group, zeros, skew, dtype):
    codes, scales, z = _matrices(E, N, K, group, zeros, dtype, T + E)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(K), device=DEV).to(dtype)
    off, row_pair, experts, sources = _routed(T, k, E, T, skew)
    for swiglu in (False, True) if N % 2 == 0 else (False,):
        got = binding.quant_product(codes, scales, x, group, zeros=z, expert_off=off, row_pair=row_pair, pairs_per_token=k,
                                    swiglu=swiglu)
        _check(got, *_want(codes, scales, z, group, x, experts, sources, swiglu))
    rows = x[torch.tensor(sources, device=DEV)]                # rows already in expert order: no row_pair
    again = binding.quant_product(codes, scales, rows, group, zeros=z, expert_off=off)
    _check(again, *_want(codes, scales, z, group, rows, experts, list(range(len(experts))), False))


def test_dropped_pairs_leave_their_rows_alone_and_strides_are_followed():
    T, k, E, N, K, group = 9, 4, 8, 48, 288, 32
    codes, scales, z = _matrices(E, N, K, group, True, BF16, 1)
    g = torch.Generator(device=DEV).manual_seed(2)
    idx = torch.rand((T, E), generator=g, device=DEV).topk(k, dim=1).indices.to(torch.int32)
    idx[::2, 1] = -1
    idx[5] = E
    off, _, row_pair = binding.sort_pairs(idx, E)
    o = off.tolist()
    f = o[-1]
    experts = [e for e in range(E) for _ in range(o[e], o[e + 1])]
    sources = [p // k for p in row_pair.tolist()[:f]]
    for pad, at in ((16, 8), (5, 3)):
        x = torch.randn((T, K + pad), generator=g, device=DEV).to(BF16)[:, at:at + K]
        out = torch.randn((T * k, N + pad), generator=g, device=DEV).to(BF16)
        kept = out.clone()
        binding.quant_product(codes, scales, x, group, zeros=z, expert_off=off, row_pair=row_pair, pairs_per_token=k,
                              out=out[:, at:at + N])
        _check(out[:f, at:at + N], *_want(codes, scales, z, group, x, experts, sources, False))
        kept[:f, at:at + N] = out[:f, at:at + N]
        assert torch.equal(out, kept)
    empty = torch.zeros(E + 1, dtype=torch.int32, device=DEV)   # no expert has a row
    out = torch.ones((T * k, N), dtype=BF16, device=DEV)
    binding.quant_product(codes, scales, torch.zeros((T, K), dtype=BF16, device=DEV), group, zeros=z, expert_off=empty,
                          row_pair=row_pair, pairs_per_token=k, out=out)
    assert (out == 1).all()


def test_values_of_every_size():
    """Tokens whose values span the type's range, infinities and NaN: each stays in its own row."""
    N, K, group = 32, 256, 64
    codes, scales, z = _matrices(1, N, K, group, True, F32, 5)
    x = torch.randn((6, K), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV)
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3, :128] *= 1e-12
    x[4] = 0
    for dtype in (BF16, F32):
        t = x.to(dtype)
        want, err = _want(codes, scales, z, group, t, [0] * 6, list(range(6)), False)
        got = binding.quant_product(codes, scales, t, group, zeros=z)
        _check(got, want, err)
        t2 = t.clone()
        t2[0, 3], t2[5, 9] = float("inf"), float("nan")
        got2 = binding.quant_product(codes, scales, t2, group, zeros=z)
        assert torch.equal(got2[1:5], got[1:5])
        assert not torch.isfinite(got2[0]).any() and torch.isnan(got2[5]).all()


@pytest.mark.parametrize("mean", [0.0, 1.0])
@pytest.mark.parametrize("K,group,zeros", [(1056, 32, True), (7168, 128, False), (2048, 64, True)])
def test_fp32_products_keep_fp32_accuracy(K, group, zeros, mean):
    """The error of all products together (2-norm, relative to the result's, or to that of independent terms where the
    tokens have a mean).  A product is a sum of n = K / 16 matrix steps of two parts and G scalings; each may be off by a unit, 2^-23, of a partial sum no larger than the result's
    scale.  Taken as independent and uniform that is sqrt(n / 3) 2^-23; a path that drops bits of the operands or of the
    sums lies far above it."""
    N, T = 512, 24
    codes, scales, z = _matrices(1, N, K, group, zeros, F32, 21)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(22), device=DEV) + mean
    got = binding.quant_product(codes, scales, x, group, zeros=z).double()
    w = _widened(codes[0], scales[0], None if z is None else z[0], group, K)
    want = x.double() @ w.T
    size = want.norm() if mean == 0 else (x.double() ** 2 @ (w ** 2).T).sqrt().norm()
    n = 2 * K / 16 + scales.shape[2]
    assert (got - want).norm() <= (n / 3) ** 0.5 * 2.0 ** -23 * size


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("zeros", [False, True])
def test_an_infinity_meets_the_weights_sign(zeros, dtype):
    """A product with one infinity is an infinity of the weight's sign, or NaN where the weight is 0."""
    N, K, group = 200, 256, 32
    codes, scales, z = _matrices(1, N, K, group, zeros, BF16, 11)
    x = torch.randn((3, K), generator=torch.Generator(device=DEV).manual_seed(12), device=DEV).to(dtype)
    clean = binding.quant_product(codes, scales, x, group, zeros=z)
    x[1, 77] = float("-inf")
    got = binding.quant_product(codes, scales, x, group, zeros=z)
    w = _widened(codes[0], scales[0], None if z is None else z[0], group, K)[:, 77]
    assert (w == 0).any() and (w > 0).any() and (w < 0).any()
    assert torch.isnan(got[1][w == 0]).all()
    assert (got[1][w > 0] == float("-inf")).all() and (got[1][w < 0] == float("inf")).all()
    assert torch.equal(got[[0, 2]], clean[[0, 2]])


def test_sources_outside_x_count_as_zero():
    N, K, group = 16, 64, 32
    codes, scales, _ = _matrices(2, N, K, group, False, BF16, 7)
    x = torch.randn((3, K), device=DEV).to(BF16)
    off = torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV)
    row_pair = torch.tensor([0, 99, -5, 2, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    got = binding.quant_product(codes, scales, x, group, expert_off=off, row_pair=row_pair)
    _check(got, *_want(codes, scales, None, group, x, [0, 0, 0, 1, 1], [0, -1, -1, 2, -1], False))
    assert (got[[1, 2, 4]] == 0).all()


def test_offsets_beyond_the_rows_are_cut():
    """expert_off entries past n_rows or out of order reach no row outside [0, n_rows)."""
    N, K, group = 16, 64, 32
    codes, scales, _ = _matrices(3, N, K, group, False, BF16, 8)
    x = torch.randn((4, K), device=DEV).to(BF16)
    off = torch.tensor([-3, 2, 1, 900], dtype=torch.int32, device=DEV)
    out = torch.zeros((8, N), dtype=BF16, device=DEV)
    binding.quant_product(codes, scales, x, group, expert_off=off, out=out[:4])
    torch.cuda.synchronize()
    assert (out[4:] == 0).all()


def test_captured_product_follows_new_routing_and_two_graphs_share_nothing():
    T, k, E, N, K, group = 12, 4, 32, 64, 640, 128
    codes, scales, z = _matrices(E, N, K, group, True, BF16, 9)

    def fill(seed):
        off, row_pair, _, _ = _routed(T, k, E, seed)
        return {"x": torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(BF16),
                "off": off, "row_pair": row_pair}

    def step(s):
        return binding.quant_product(codes, scales, s["x"], group, zeros=z, expert_off=s["off"], row_pair=s["row_pair"],
                                     pairs_per_token=k)

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
        assert torch.equal(got, step(s))


def test_wrapper_refuses_what_does_not_fit():
    codes, scales, z = _matrices(2, 16, 64, 32, True, BF16, 1)
    x = torch.zeros((4, 64), dtype=BF16, device=DEV)
    off, pairs = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV), torch.arange(4, dtype=torch.int32, device=DEV)
    q = binding.quant_product
    bad = [lambda: q(codes, scales, x, 16, expert_off=off), lambda: q(codes, scales, x, 0, expert_off=off), lambda: q(codes, scales, x, 32),
           lambda: q(codes, scales, x.half(), 32, expert_off=off), lambda: q(codes, scales.half(), x, 32, expert_off=off),
           lambda: q(codes, scales, x, 64, expert_off=off), lambda: q(codes, scales, x[:, :32], 32, expert_off=off),
           lambda: q(codes, scales, x, 32, zeros=z[:1], expert_off=off), lambda: q(codes, scales, x, 32, expert_off=off[:2]),
           lambda: q(codes[:, :15].contiguous(), scales[:, :15].contiguous(), x, 32, expert_off=off, swiglu=True),
           lambda: q(codes, scales, x, 32, expert_off=off, row_pair=pairs, pairs_per_token=0),
           lambda: q(codes, scales, x, 32, expert_off=off.long()), lambda: q(codes, scales, x.cpu(), 32, expert_off=off),
           lambda: q(codes[:1, :, :8].contiguous(), scales[:1, :, :1].contiguous(), x[:, :16].contiguous(), 32)]
    for call in bad:
        with pytest.raises(binding.DeaMoEError):
            call()


def test_matrices_beyond_32_bit_offsets():
    """5 GB of codes: the products of the last experts against their definition."""
    E, N, K, group, T = 288, 4096, 8704, 128, 3
    codes = torch.empty((E, N, K // 2), dtype=torch.uint8, device=DEV)
    for e in range(E):
        codes[e].random_(0, 256, generator=torch.Generator(device=DEV).manual_seed(e))
    assert codes.numel() > 2 ** 32
    scales = torch.rand((E, N, K // group), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).mul_(0.01).to(BF16)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(BF16)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    off[E - 1] = 1
    off[E] = T
    got = binding.quant_product(codes, scales, x, group, expert_off=off)
    _check(got, *_want(codes, scales, None, group, x, [E - 2, E - 1, E - 1], [0, 1, 2], False))


@pytest.mark.parametrize("captured", [False, True])
def test_product_without_rows_is_over_when_its_call_is(captured):
    """No expert has a row: the workspace is the caller's again, and stays what the next kernel of the stream makes it."""
    E, N, K, group, T = 4, 64, 16384, 32, 4096
    codes, scales, _ = _matrices(E, N, K, group, False, F32, 31)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(32), device=DEV)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    out = torch.full((T, N), 7.0, device=DEV)
    L, p = binding.lib(), binding._dptr
    need = L.deamoe_quant_workspace(binding.F32, T, K)
    workspace = torch.empty(need, dtype=torch.uint8, device=DEV)

    def step():
        assert L.deamoe_quant_product(binding._stream(), binding.F32, p(codes), binding.F32, p(scales), None, E, N, K, group, p(x), K,
                                      T, p(off), None, 1, T, 0, p(out), N, p(workspace), need) == binding.OK
        workspace.fill_(0xa5)

    step()
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for _ in range(20):
        workspace.zero_()
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert (workspace == 0xa5).all() and (out == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
@pytest.mark.parametrize("large", [1e4, 1e6, 1e12, 1e30, 3e38])
def test_small_values_keep_their_bits_beside_a_large_one_of_weight_zero(large, group, zeros, dtype):
    """The bound is relative to the products, of which the large value's is 0: the others are as exact as without it."""
    N, K, T = 96, 1408, 11
    codes, scales, z = _matrices(1, N, K, group, zeros, F32, 41)
    at = [5, 130, 1407]                                        # columns of either nibble, of the first and the last group
    for c in at:
        zero = torch.full((N,), 8, dtype=torch.uint8, device=DEV) if z is None else z[0, :, c // group]
        old = codes[0, :, c // 2]
        codes[0, :, c // 2] = (old & 15) | zero << 4 if c & 1 else (old & 240) | zero
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(42), device=DEV)
    x[:, at[0]], x[::2, at[1]], x[1:9, at[2]] = large, -large, large
    x = x.to(dtype)
    assert torch.isfinite(x).all()
    got = binding.quant_product(codes, scales, x, group, zeros=z)
    _check(got, *_want(codes, scales, z, group, x, [0] * T, list(range(T)), False))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_at_the_ends_of_the_range(dtype):
    """Rows whose products with the codes alone would overflow, and rows of subnormal values: results that the type can hold
    are held.  A result's subnormal operands count in full: the bound has no absolute part."""
    N, K, group, T = 48, 32, 32, 6
    codes, _, z = _matrices(1, N, K, group, True, F32, 43)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(44), device=DEV).clamp(-3, 3)
    for size, scale in ((1e38, 2.0 ** -12), (2.0 ** 96, 1.0), (2.0 ** -120, 2.0 ** 40), (2.0 ** -126, 2.0 ** 60)):
        t = (x * size).to(dtype)
        scales = torch.full((1, N, 1), scale, device=DEV)
        want, err = _want(codes, scales, z, group, t, [0] * T, list(range(T)), False)
        got = binding.quant_product(codes, scales, t, group, zeros=z)
        assert torch.isfinite(got).all()
        half = torch.finfo(dtype).eps / 2
        assert ((got.double() - want).abs() <= err + half * (want.abs() + err)).all(), size


@pytest.mark.parametrize("off", [[0, 64, 0, 64, 64], [0, 10, 9, 20, 64], [64, 0, 0, 0, 0], [0, 0, 0, 70, 69 - 64]])
def test_offsets_that_decrease_write_nothing(off):
    """Ranges that overlap could hold more rows in all than n_rows, which is what the kernel's counting is sized by."""
    N, K, group, R = 48, 64, 32, 64
    codes, scales, _ = _matrices(4, N, K, group, False, BF16, 51)
    x = torch.randn((R, K), device=DEV).to(BF16)
    out = torch.full((R, N), 5.0, dtype=BF16, device=DEV)
    binding.quant_product(codes, scales, x, group, expert_off=torch.tensor(off, dtype=torch.int32, device=DEV), out=out)
    assert (out == 5).all()


# Rows of an expert: none, one, around passes of 8 and 16 tokens, several passes
COUNTS = [5, 12, 40, 0, 1, 8, 9, 16, 17, 3, 2, 0, 24, 33, 7, 15]


def _in_expert_order(counts, k, seed):
    off = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    R = sum(counts)
    pairs = torch.randperm(R, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    return off, pairs.to(torch.int32), [e for e, c in enumerate(counts) for _ in range(c)], [p // k for p in pairs.tolist()]


# Two row tiles a warp (296 and more of them to share): 628 SwiGLU columns and 1256 rows are no multiple of the 32-row tile,
# which then overlaps the one before; 2080 columns end inside a step, 1120 inside a group of 64 or 128
@pytest.mark.parametrize("swiglu", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros,sdtype", [(False, BF16), (True, BF16), (True, F32)])
@pytest.mark.parametrize("N,K", [(1256, 2080), (1300, 1120)])
def test_two_tiles_a_warp(N, K, zeros, sdtype, group, dtype, swiglu):
    k = 8
    off, pairs, experts, sources = _in_expert_order(COUNTS, k, N)
    codes, scales, z = _matrices(len(COUNTS), N, K, group, zeros, sdtype, K)
    x = torch.randn((-(-sum(COUNTS) // k), K), generator=torch.Generator(device=DEV).manual_seed(K), device=DEV).to(dtype)
    got = binding.quant_product(codes, scales, x, group, zeros=z, expert_off=off, row_pair=pairs, pairs_per_token=k, swiglu=swiglu)
    _check(got, *_want(codes, scales, z, group, x, experts, sources, swiglu))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("E,N,K", [(40, 4096, 2048), (80, 4096, 768), (160, 4096, 512)])
def test_fewer_warps_a_tile(E, N, K, zeros, dtype):
    """So many items that 4, 2 or 1 of a block's warps share a tile's columns: the main form of a decode step over experts."""
    counts = [1 + (7 * e) % 19 if e % 8 == 0 else 1 + e % 3 for e in range(E)]
    off, _, experts, _ = _in_expert_order(counts, 1, 1)
    codes, scales, z = _matrices(E, N, K, 128, zeros, BF16, E)
    x = torch.randn((sum(counts), K), generator=torch.Generator(device=DEV).manual_seed(K), device=DEV).to(dtype)
    got = binding.quant_product(codes, scales, x, 128, zeros=z, expert_off=off, swiglu=True)
    _check(got, *_want(codes, scales, z, 128, x, experts, list(range(len(experts))), True))


@pytest.mark.parametrize("large", [0.0, 1e6, 1e20])
@pytest.mark.parametrize("K,group,zeros", [(1056, 32, True), (7168, 128, False), (2048, 64, True)])
def test_fp32_products_round_only_their_sums(K, group, zeros, large):
    """The error of all products together, 2-norm.  Of zero-mean terms a partial sum's square is the share of its terms in the
    result's, half of that on average.  On a group's sum (share group / K) there are two matrix steps in 32 columns, which
    cut: a unit of 2^-23, a third of its square.  On the whole sum there are G scalings, which round: a twelfth.  So the
    squares add up to (K / 16) (group / K) / 6 + G / 24 squared units.  A large value that meets weights of 0 adds nothing."""
    N, T = 512, 24
    codes, scales, z = _matrices(1, N, K, group, zeros, F32, 61)
    x = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(62), device=DEV)
    if large:
        for c in (3, 700):
            zero = torch.full((N,), 8, dtype=torch.uint8, device=DEV) if z is None else z[0, :, c // group]
            old = codes[0, :, c // 2]
            codes[0, :, c // 2] = (old & 15) | zero << 4 if c & 1 else (old & 240) | zero
            x[:, c] = large
    got = binding.quant_product(codes, scales, x, group, zeros=z).double()
    want = x.double() @ _widened(codes[0], scales[0], None if z is None else z[0], group, K).T
    assert (got - want).norm() <= (group / 96 + scales.shape[2] / 24) ** 0.5 * 2.0 ** -23 * want.norm()
