"""The operators around a layer run together, as a model's block uses them: a decode step over 4-bit experts, routed by the
library's router, and a training step with its gradients."""
import numpy as np
import pytest
import torch

from oracle import ref
from paper_2608_14385_b200 import binding, synth
from tests.bounds import Bounded
from tests.common import oracle_cfg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32
SHAPE = synth.LayerShape("block", hidden=512, n_dept=4, experts_per_dept=8, ffn=192, priv=64, top_k=4, act_dtype=0)


def _g(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _gauss(shape, seed, scale=1.0, mean=0.0):
    return torch.randn(shape, generator=_g(seed), device=DEV) * scale + mean


def _experts(E, n_out, n_in, group, seed):
    codes = torch.randint(0, 256, (E, n_out, n_in // 2), generator=_g(seed), device=DEV, dtype=torch.uint8)
    scales = torch.rand((E, n_out, -(-n_in // group)), generator=_g(seed + 1), device=DEV) * 0.01 + 0.002
    zeros = torch.randint(6, 10, scales.shape, generator=_g(seed + 2), device=DEV, dtype=torch.uint8)
    q = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).double()
    col = torch.arange(n_in, device=DEV) // group
    return codes, scales, zeros, (q - zeros.double()[..., col]) * scales.double()[..., col]


def _decode(s):
    """One decode step of a block: every intermediate, in the order in which it is made."""
    u = binding.norm(s["x"], s["w_pre"], 1e-6)
    idx, w = binding.route_static(s["router"], u, SHAPE.n_dept, SHAPE.experts_per_dept, SHAPE.top_k)
    off, pair_row, row_pair = binding.sort_pairs(idx, s["E"])
    y = binding.quant_product(*s["up"][:2], u, 64, zeros=s["up"][2], expert_off=off, row_pair=row_pair, pairs_per_token=SHAPE.top_k,
                              swiglu=True)
    z = binding.quant_product(*s["down"][:2], y, 32, zeros=s["down"][2], expert_off=off)
    o = binding.combine(z, pair_row, w)
    out, nxt = binding.norm_residual(s["x"], o, s["w_post"], 1e-6, next_weight=s["w_next"])
    return u, idx, w, off, pair_row, row_pair, y, z, o, out, nxt


def _state(T, seed):
    h, f, E = SHAPE.hidden, SHAPE.ffn, SHAPE.n_dept * SHAPE.experts_per_dept
    return {"E": E, "x": _gauss((T, h), seed), "router": _gauss((E, h), 2, 0.05), "w_pre": _gauss((h,), 3, 0.1, 1.0),
            "w_post": _gauss((h,), 4, 0.1, 1.0), "w_next": _gauss((h,), 5, 0.1, 1.0),
            "up": _experts(E, 2 * f, h, 64, 10), "down": _experts(E, h, f, 32, 20)}


@pytest.mark.parametrize("T", [1, 7, 40])
def test_decode_step_over_four_bit_experts(T):
    """Each stage against its definition in 64 bits on the inputs that it got, the routing against the oracle."""
    s = _state(T, T)
    u, idx, w, off, pair_row, row_pair, y, z, o, out, nxt = _decode(s)
    X = Bounded(s["x"])
    inv = lambda v: ((v * v).sum(1, keepdim=True) * Bounded(1.0 / SHAPE.hidden) + Bounded(1e-6)).rsqrt()  # noqa: E731
    (X * inv(X) * Bounded(s["w_pre"])).within(u, "norm")
    want = ref.route(oracle_cfg(SHAPE), s["router"].cpu().numpy(), u.cpu().numpy(), want_logits=True)
    safe = want["gap"] > 1e-5 * np.abs(want["logits"]).max(axis=1)
    assert safe.all(), "seed too close to a routing tie"
    assert (idx.cpu().numpy() == want["idx"]).all()
    o_list = off.tolist()
    assert o_list[-1] == T * SHAPE.top_k
    expert = [e for e in range(s["E"]) for _ in range(o_list[e], o_list[e + 1])]
    token = (row_pair.long() // SHAPE.top_k).tolist()
    U, Y = u.double(), y.double()
    K = SHAPE.hidden
    # a sum of n products and 2 G scalings, each addition good to one unit; then SiLU's roundings (see the product's own tests)
    for r in range(T * SHAPE.top_k):
        W = s["up"][3][expert[r]]
        v, e = W @ U[token[r]], (K + 2 * s["up"][1].shape[2] + 8) * 2.0 ** -23 * (W.abs() @ U[token[r]].abs())
        f = SHAPE.ffn
        silu = v[:f] * torch.sigmoid(v[:f])
        es = 1.1 * e[:f] + 8 * 2.0 ** -24 * (silu.abs() + 1.1 * e[:f])
        got, bound = silu * v[f:], (silu.abs() + es) * e[f:] + es * v[f:].abs() + 2 * 2.0 ** -24 * (silu * v[f:]).abs()
        assert ((y[r].double() - got).abs() <= bound).all()
        W = s["down"][3][expert[r]]
        got, bound = W @ Y[r], (f + 2 * s["down"][1].shape[2] + 9) * 2.0 ** -23 * (W.abs() @ Y[r].abs())
        assert ((z[r].double() - got).abs() <= bound).all()
    (Bounded(z[pair_row.long()]) * Bounded(w[:, :, None].double().expand(T, SHAPE.top_k, K))).sum(1).within(o, "combine")
    O = Bounded(o)  # noqa: E741
    S = X + O * inv(O) * Bounded(s["w_post"])
    S.within(out, "out")
    (S * inv(S) * Bounded(s["w_next"])).within(nxt, "next")


def test_decode_step_captured_in_a_graph_follows_new_tokens():
    s = _state(9, 1)
    _decode(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _decode(s)
    for seed in (2, 3):
        s["x"].copy_(_gauss((9, SHAPE.hidden), seed))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, _decode(s)):
            assert torch.equal(a, b)


def test_beside_a_layer_of_the_library():
    """The layer's own routing feeds the sort; the norms wrap the layer's forward; all on one stream."""
    shape = synth.LayerShape("block-layer", hidden=256, n_dept=4, experts_per_dept=4, ffn=128, priv=64, top_k=3)
    weights = synth.make_deamoe_weights(shape, 3, DEV)
    layer = binding.Layer(shape, weights, 16)
    try:
        x = synth.make_tokens(shape, 11, 4, DEV)
        w = torch.ones(shape.hidden, dtype=torch.bfloat16, device=DEV)
        u = binding.norm(x, w, 1e-6)
        idx, p = layer.route(u)
        off, pair_row, row_pair = binding.sort_pairs(idx, 16)
        out, nxt = binding.norm_residual(x, layer.forward(u), w, 1e-6, next_weight=w)
        torch.cuda.synchronize()
        state = layer.routing(11)
        assert (off.cpu().numpy() == state["expert_off"]).all()
        assert ((row_pair.cpu().numpy() // 3) == state["expert_tok"]).all()
        plain = binding.norm_residual(x, layer.forward(u), w, 1e-6, next_weight=w)
        assert torch.equal(out, plain[0]) and torch.equal(nxt, plain[1])
        assert layer.stats()["device_status"] == 0
    finally:
        layer.close()


def test_training_step_gradients_against_differences():
    """norm -> dispatch -> experts (plain matrices, 64 bits) -> combine -> gated residual with the next norm; the chain of
    backward calls along a random direction against the central difference of the whole step in 64 bits.  Step 1e-4:
    truncation below 1e-6 relative; the fp32 calls' own roundings, h 2^-24 of the terms' sizes, stay below 1e-4 of them."""
    T, k, E, h = 24, 3, 6, 96
    eps = 1e-6
    idx = torch.rand((T, E), generator=_g(1), device=DEV).topk(k, dim=1).indices.to(torch.int32)
    idx[3] = -1                                                # a padded token
    idx[5, 1] = E                                              # a dropped pair
    off, pair_row, row_pair = binding.sort_pairs(idx, E)
    f = int(off[-1])
    expert = torch.repeat_interleave(torch.arange(E, device=DEV), (off[1:] - off[:-1]).long())
    W = _gauss((E, h, h), 2, 0.1).double()
    p = {"x": _gauss((T, h), 3), "w": torch.rand((T, k), generator=_g(4), device=DEV), "w_pre": _gauss((h,), 5, 0.2, 1.0),
         "w_post": _gauss((h,), 6, 0.2, 1.0), "w_next": _gauss((h,), 7, 0.2, 1.0), "gate": _gauss((h,), 8, 0.3, 0.5)}
    along = {n: torch.randn(t.shape, generator=_g(20 + i), device=DEV).double() for i, (n, t) in enumerate(p.items())}
    dout, dnext = _gauss((T, h), 40), _gauss((T, h), 41)

    def loss(step):
        q = {n: t.double() + step * along[n] for n, t in p.items()}
        unit = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)  # noqa: E731
        u = unit(q["x"]) * q["w_pre"]
        y = torch.tanh(torch.bmm(W[expert], u[row_pair[:f].long() // k][:, :, None])[:, :, 0])
        ok = pair_row >= 0
        take = y[pair_row.long().clamp(min=0)] * ok[:, :, None]
        o = (take * q["w"][:, :, None]).sum(1)
        s = q["x"] + q["gate"] * unit(o) * q["w_post"]
        return (s * dout.double()).sum() + (unit(s) * q["w_next"] * dnext.double()).sum()

    u = binding.norm(p["x"], p["w_pre"], eps)
    rows = binding.dispatch(u, pair_row)
    pre = torch.bmm(W[expert], rows[:f].double()[:, :, None])[:, :, 0]
    y = torch.zeros_like(rows)
    y[:f] = torch.tanh(pre).float()
    o = binding.combine(y, pair_row, p["w"])
    kw = dict(gate=p["gate"], next_weight=p["w_next"])
    binding.norm_residual(p["x"], o, p["w_post"], eps, **kw)
    dx, do, dgate, dpost, dnw = binding.norm_residual_backward(p["x"], o, p["w_post"], eps, dout, du=dnext, **kw)
    dy, dw = binding.combine_backward(do, y, pair_row, p["w"])
    drows = torch.zeros_like(rows)
    drows[:f] = torch.bmm(W[expert].transpose(1, 2), (dy[:f].double() * (1 - torch.tanh(pre) ** 2))[:, :, None])[:, :, 0].float()
    du = binding.dispatch_backward(drows, pair_row)
    dx, dpre = binding.norm_backward(p["x"], p["w_pre"], eps, du, dadd=dx)
    grads = {"x": dx, "w": dw, "w_pre": dpre, "w_post": dpost, "w_next": dnw, "gate": dgate}
    # the padded token's rows are nowhere: its o and its weights' gradients are 0
    assert (o[3] == 0).all() and (dw[3] == 0).all()
    difference = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = sum((g.double() * along[n]).sum() for n, g in grads.items())
    size = sum((g.double().abs() * along[n].abs()).sum() for n, g in grads.items())
    assert abs(got - difference) <= 1e-4 * size
