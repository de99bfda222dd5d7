"""The products around a layer as a model uses them together: a prompt through its block (8-bit projection, experts, next block's
rows in 8 bits), and a training step through the experts with the gradients of all that is around them."""
import pytest
import torch

from paper_2608_14385_b200 import binding
from tests import product_bounds as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
E, K, H, F = 12, 3, 520, 264


def _gauss(shape, seed, scale=1.0, mean=0.0, dtype=BF16):
    return (torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale + mean).to(dtype)


def _routing(T, seed, drop):
    g = torch.Generator(device=DEV).manual_seed(seed)
    top = torch.randn((T, E), generator=g, device=DEV).topk(K, dim=1)
    idx = top.indices.to(torch.int32)
    if drop:
        idx[::3, 1] = -1
    return idx, torch.softmax(top.values, dim=1)


def _weights():
    return {"wgu": _gauss((E, 2 * F, H), 1, H ** -0.5), "wd": _gauss((E, H, F), 2, F ** -0.5), "proj": _gauss((H, H), 3, H ** -0.5),
            "bias": _gauss((H,), 4, 0.2), "w_post": _gauss((H,), 5, 0.1, 1.0), "w_next": _gauss((H,), 6, 0.1, 1.0)}


@pytest.mark.parametrize("T,drop", [(1, False), (5, True), (60, False), (400, True)])
def test_prompt_through_a_block(T, drop):
    """Every stage against its definition on the inputs that it got."""
    w, x = _weights(), _gauss((T, H), T, 2.0)
    idx, gate = _routing(T, T + 1, drop)
    h = 528                                                      # the projection reads 8-bit rows of whole 16-byte pieces
    x_wide, proj_wide = torch.zeros((T, h), dtype=BF16, device=DEV), torch.zeros((H, h), dtype=BF16, device=DEV)
    x_wide[:, :H], proj_wide[:, :H] = x, w["proj"]
    p8, sp = binding.norm_quant(proj_wide, None, 1e-6, normalise=False)
    u8, su = binding.norm_quant(x_wide, None, 1e-6)
    y = binding.product(u8, p8, bias=w["bias"], act=binding.SIGMA_SILU, residual=x, x_scale=su, weight_scale=sp)
    z, e = pb.dot(u8.double(), None, p8.double(), None)
    s = su.double()[:, None] * sp.double()[None, :]
    z, e = pb.times(z, e, s, s * pb.UNIT)
    z, e = pb.act(1, *pb.plus(z, e, w["bias"].double()[None, :], torch.zeros_like(z)))
    pb.check(y, *pb.plus(z, e, x.double(), torch.zeros_like(z)), "projection")

    off, pair_row, row_pair = binding.sort_pairs(idx, E)
    rows = binding.dispatch(y, pair_row)
    o = binding.ffn(rows, w["wgu"], w["wd"], expert_off=off)
    at = off.tolist()
    for i in range(E):
        if at[i + 1] > at[i]:
            pb.check(o[at[i]:at[i + 1]], *pb.ffn(rows[at[i]:at[i + 1]].double(), w["wgu"][i].double(), w["wd"][i].double())[0], f"expert {i}")
    b = binding.combine(o, pair_row, gate)
    out, codes, scale = binding.norm_residual_quant(y, b, w["w_post"], 1e-6, next_weight=w["w_next"])
    plain, nxt = binding.norm_residual(y, b, w["w_post"], 1e-6, next_weight=w["w_next"])
    # the same sum and the same norm, once as bf16 and once as codes: a code is off by 2^-4 of its value at most (2^-10 of the row's
    # largest where it is subnormal), the bf16 value by 2^-8, the fp32 arithmetic of either by far less
    assert torch.equal(out, plain)
    back = codes.float() * scale[:, None]
    assert ((back - nxt.float()).abs() <= nxt.float().abs() * (2.0 ** -4 + 2.0 ** -8) * 1.01 + scale[:, None] * 2.0 ** -10 * 1.01).all()
    assert binding.operator_status() == binding.OK


def _train(w, x, idx, gate, dout):
    """out = x + b, b the experts' sum of silu(x P^T + bias); all gradients, by the library."""
    y = binding.product(x, w["proj"], bias=w["bias"], act=binding.SIGMA_SILU)
    off, pair_row, _ = binding.sort_pairs(idx, E)
    rows = binding.dispatch(y, pair_row)
    o = binding.ffn(rows, w["wgu"], w["wd"], expert_off=off)
    out = binding.combine(o, pair_row, gate)
    do, dgate = binding.combine_backward(dout, o, pair_row, gate)
    drows, dwgu, dwd = binding.ffn_backward(rows, w["wgu"], w["wd"], do, expert_off=off)
    dy = binding.dispatch_backward(drows, pair_row)
    dx, dproj, dbias = binding.product_backward(x, w["proj"], dy, bias=w["bias"], act=binding.SIGMA_SILU)
    return out, dgate, dwgu, dwd, dx, dproj, dbias


@pytest.mark.parametrize("T,drop", [(4, False), (90, True), (300, False)])
def test_training_step_against_the_definition(T, drop):
    """The chain's gradients against those of its definition in 64 bits, differentiated by torch, in 2-norm.  A chain of n roundings
    to bf16, each 2^-8 of a value at most and independent of the others, is off by no more than n 2^-8 of the norm (the
    maps between them keep relative norms but for the cancellation in sums of random terms, which does the same to the result);
    there are 11 of them from the input to the last gradient."""
    w, x, dout = _weights(), _gauss((T, H), T), _gauss((T, H), T + 1)
    idx, gate = _routing(T, T + 2, drop)
    got = _train(w, x, idx, gate, dout)
    leaf = {n: w[n].double().requires_grad_() for n in ("wgu", "wd", "proj", "bias")}
    X, G = x.double().requires_grad_(), gate.double().requires_grad_()
    y = torch.nn.functional.silu(X @ leaf["proj"].T + leaf["bias"])
    out = torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for q in range(K):
        for i in range(E):
            t = (idx[:, q] == i).nonzero()[:, 0]
            if len(t):
                z = y[t] @ leaf["wgu"][i].T
                r = (torch.nn.functional.silu(z[:, :F]) * z[:, F:]) @ leaf["wd"][i].T
                out = out.index_add(0, t, r * G[t, q][:, None])
    want = torch.autograd.grad(out, [G, leaf["wgu"], leaf["wd"], X, leaf["proj"], leaf["bias"]], dout.double())
    for name, a, b in zip(("out", "gate", "gate / up", "down", "x", "projection", "bias"), got, (out.detach(),) + want):
        assert (a.double() - b).norm() <= 11 * 2.0 ** -8 * b.norm(), (name, ((a.double() - b).norm() / b.norm()).item())


def test_training_step_captured_while_an_eager_graph_of_the_same_leaves_lives():
    w, T = _weights(), 70
    x, dout = _gauss((T, H), 1), _gauss((T, H), 2)
    idx, gate = _routing(T, 3, True)
    leaf = x.clone().requires_grad_()
    alive = torch.nn.functional.silu(leaf @ w["proj"].T)         # torch's own graph of a leaf that shares the step's memory
    want = _train(w, leaf.detach(), idx, gate, dout)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = _train(w, leaf.detach(), idx, gate, dout)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    alive.sum().backward()
    assert torch.isfinite(leaf.grad).all()


def test_what_the_kernel_before_wrote_is_seen_and_what_comes_after_sees_all():
    """The calls' kernels are launched before the kernel in front of them has ended: inputs and weights that it writes must be
    read after it, and the kernel behind must find every output."""
    T = 300
    sets = [{"x": _gauss((T, H), i), "w": _gauss((H, H), 10 + i, H ** -0.5), "wgu": _gauss((E, 2 * F, H), 20 + i, H ** -0.5),
             "wd": _gauss((E, H, F), 30 + i, F ** -0.5), "dy": _gauss((T, H), 40 + i)} for i in range(2)]
    off = torch.tensor([0, 9, 9, 60, 61, 100, 130, 131, 140, 200, 260, 290, 300], dtype=torch.int32, device=DEV)
    big = torch.empty(1 << 24, device=DEV)

    def calls(s):
        return [binding.product(s["x"][:5], s["w"]), binding.product(s["x"], s["w"], act=binding.SIGMA_GELU), binding.product(s["x"][:40], s["w"]),
                binding.ffn(s["x"][:7], s["wgu"][:1], s["wd"][:1]), binding.ffn(s["x"], s["wgu"], s["wd"], expert_off=off),
                *binding.ffn_backward(s["x"], s["wgu"], s["wd"], s["dy"], expert_off=off),
                *binding.product_backward(s["x"], s["w"], s["dy"], act=binding.SIGMA_SILU)[:2]]

    want = [[t.clone() for t in calls(s)] for s in sets]
    now = {n: torch.empty_like(t) for n, t in sets[0].items()}
    wrong = []
    for i in range(40):
        s = sets[i % 2]
        big.fill_(float(i))                                       # keeps the device busy until the copies' turn comes
        for n, t in now.items():
            t.copy_(s[n])
        wrong.append([(a != b).sum() for a, b in zip(calls(now), want[i % 2])])
        now["w"].zero_()                                          # one call right behind the kernels that write its weights
        now["w"].copy_(s["w"])
        wrong.append([(binding.product(now["x"][:5], now["w"]) != want[i % 2][0]).sum()])
    assert all(int(n) == 0 for w in wrong for n in w)
