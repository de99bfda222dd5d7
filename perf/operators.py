"""Cases and plain forms of the operators around a layer: tokens sorted by expert and back, the norms of the block,
products with 4-bit expert matrices.

`own` selects what `run` does: False computes the operator from elementary torch operations in 32 bits, True calls the
library (paper_2608_14385_b200.binding).  Both take the state that `prepare` makes on the current CUDA device.

Operators, as a user calls them:
  tokens           sort_pairs, dispatch (rows in expert order), combine (back, with the gate weights)
  tokens_backward  dispatch_backward and combine_backward: the gradients of the same step
  norms            norm before the block, norm_residual after it (with the next block's norm in the same pass)
  norms_backward   norm_residual_backward and norm_backward
  quant            quant_product: matrix-vector products with 4-bit weights, one matrix or the active experts'
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6

# Sizes: hidden 7168, 256 experts, top-8, ffn 2048 is the DeepSeek-V3 shape of synth.py; hidden 4096, ffn 1408 its 7b
# shape; hidden 1024, 672 experts, top-10, ffn 384 its b7-paper shape; hidden 7168, 864 experts, top-10 its dsv3-paper
# shape.  Odd sizes are generic.


def listed():
    return [
        # one decode step of the DeepSeek-V3 shape: latency of three small launches
        dict(name="tokens decode 16", op="tokens", tokens=16, hidden=7168, experts=256, top_k=8, drop=0.0, type="bf16"),
        # a prompt of 4096 tokens on the same shape: all bytes
        dict(name="tokens prompt 4096", op="tokens", tokens=4096, hidden=7168, experts=256, top_k=8, drop=0.0, type="bf16"),
        # odd sizes, fp32, a tenth of the pairs dropped (experts of another rank, padding): training on a small model
        dict(name="tokens ragged fp32", op="tokens", tokens=1021, hidden=1027, experts=672, top_k=10, drop=0.1, type="fp32"),
        # the gradients of a training step of 4096 tokens
        dict(name="tokens gradient 4096", op="tokens_backward", tokens=4096, hidden=7168, experts=256, top_k=8, drop=0.0, type="bf16"),
        # the same of a small fp32 model with dropped pairs
        dict(name="tokens gradient fp32", op="tokens_backward", tokens=777, hidden=1024, experts=672, top_k=10, drop=0.1, type="fp32"),
        # one decode step of 8 tokens on the 7b shape, norm before and after, no gate
        dict(name="norms decode 8", op="norms", tokens=8, hidden=4096, gate="none", type="bf16"),
        # a prompt of 8192 tokens, a learned gate per channel
        dict(name="norms prompt 8192", op="norms", tokens=8192, hidden=7168, gate="channel", type="bf16"),
        # the gradients of a training step of 4096 tokens, gate per channel
        dict(name="norms gradient 4096", op="norms_backward", tokens=4096, hidden=7168, gate="channel", type="bf16"),
        # odd sizes, fp32, one gate value per token
        dict(name="norms gradient fp32", op="norms_backward", tokens=333, hidden=1027, gate="token", type="fp32"),
        # one token through one shared expert's gate and up matrices, with the SwiGLU: the smallest product
        dict(name="quant one token", op="quant", experts=1, rows=4096, cols=7168, group=128, zeros=False, tokens=1, top_k=1,
             swiglu=True, type="bf16"),
        # 16 tokens through the gate and up matrices of their top-8 of 256 experts, DeepSeek-V3 shape
        dict(name="quant experts 16", op="quant", experts=256, rows=4096, cols=7168, group=128, zeros=False, tokens=16,
             top_k=8, swiglu=True, type="bf16"),
        # odd sizes, small groups, zero points, fp32 tokens, several tokens an expert
        dict(name="quant ragged fp32", op="quant", experts=16, rows=1003, cols=1056, group=32, zeros=True, tokens=37, top_k=2,
             swiglu=False, type="fp32"),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tokens", "tokens_backward", "norms", "norms_backward", "quant", "quant"])
    kind = rng.choice(["bf16", "bf16", "fp32"])
    hidden = rng.choice([_between(rng, 64, 7168), 8 * _between(rng, 8, 896), 256 * rng.randint(1, 28)])
    if op.startswith("tokens"):
        experts = _between(rng, 8, 1024)
        top_k = rng.randint(1, min(10, experts))
        most = 4096 * 8 * 7168 // (hidden * top_k * (2 if kind == "fp32" else 1))
        return dict(op=op, tokens=_between(rng, 1, max(1, min(16384, most))), hidden=hidden, experts=experts, top_k=top_k,
                    drop=rng.choice([0.0, 0.0, 0.1, 0.6]), type=kind)
    if op.startswith("norms"):
        most = (8192 if op == "norms" else 4096) * 7168 // (hidden * (2 if kind == "fp32" else 1))
        return dict(op=op, tokens=_between(rng, 1, max(1, min(16384, most))), hidden=hidden,
                    gate=rng.choice(["none", "channel", "token", "full"]), type=kind)
    experts = rng.choice([1, _between(rng, 2, 256)])
    top_k = 1 if experts == 1 else rng.randint(1, min(8, experts))
    rows, cols = 2 * _between(rng, 64, 2048), 32 * _between(rng, 4, 224)
    tokens = _between(rng, 1, 32)
    while tokens * top_k > 128:
        tokens = (tokens + 1) // 2
    return dict(op=op, experts=experts, rows=rows, cols=cols, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5,
                tokens=tokens, top_k=top_k, swiglu=rng.random() < 0.5, type=kind)


# ---------------------------------------------------------------- inputs

def _routing(g, tokens, experts, top_k, drop):
    """Top-k of Gaussian logits (experts of a token in order of decreasing logit) and softmax weights over them; a share
    `drop` of the pairs marked -1."""
    logits = torch.randn((tokens, experts), generator=g, device="cuda")
    top = torch.topk(logits, top_k, dim=1)
    idx = top.indices.to(torch.int32)
    w = torch.softmax(top.values, dim=1)
    if drop > 0:
        idx = torch.where(torch.rand((tokens, top_k), generator=g, device="cuda") < drop, torch.full_like(idx, -1), idx)
    return idx, w


def _sorted(idx, experts):
    """Rows in expert order, ties in pair order: first row of each expert, row of each pair, pair of each row."""
    flat = idx.reshape(-1).long()
    ok = (flat >= 0) & (flat < experts)
    key = torch.where(ok, flat, torch.full_like(flat, experts))
    order = torch.sort(key, stable=True).indices
    count = torch.zeros(experts + 1, dtype=torch.long, device=idx.device).scatter_add_(0, key, torch.ones_like(key))
    off = torch.cat([torch.zeros_like(count[:1]), torch.cumsum(count[:experts], 0)])
    at = torch.arange(flat.numel(), device=idx.device)
    filled = at < off[-1]
    pair_row = torch.empty_like(at)
    pair_row[order] = torch.where(filled, at, torch.full_like(at, -1))
    row_pair = torch.where(filled, order, torch.full_like(order, -1))
    return off.to(torch.int32), pair_row.to(torch.int32).view(idx.shape), row_pair.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t = TYPES[case["type"]]

    def gauss(*shape, scale=1.0, mean=0.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(mean).to(t)

    op, s = case["op"], {"case": case}
    if op in ("tokens", "tokens_backward"):
        T, h, k = case["tokens"], case["hidden"], case["top_k"]
        s["idx"], s["w"] = _routing(g, T, case["experts"], k, case["drop"])
        s["y"] = gauss(T * k, h)
        s["rows"] = torch.zeros((T * k, h), dtype=t, device="cuda")
        if op == "tokens":
            s["x"] = gauss(T, h)
        else:
            s["pair_row"] = _sorted(s["idx"], case["experts"])[1]
            s["dout"] = gauss(T, h)
            s["drows"] = gauss(T * k, h)
        return s
    if op in ("norms", "norms_backward"):
        T, h = case["tokens"], case["hidden"]
        s["x"], s["y"] = gauss(T, h, scale=2.0), gauss(T, h, scale=0.5)
        for name in ("w_pre", "w_post", "w_next"):
            s[name] = gauss(h, scale=0.2, mean=1.0)
        shape = {"none": None, "channel": (h,), "token": (T,), "full": (T, h)}[case["gate"]]
        s["gate"] = None if shape is None else gauss(*shape, scale=0.3, mean=0.5)
        if op == "norms_backward":
            s["dout"], s["du"], s["dh"] = gauss(T, h), gauss(T, h), gauss(T, h)
        return s
    E, N, K, T, k = case["experts"], case["rows"], case["cols"], case["tokens"], case["top_k"]
    G = -(-K // case["group"])
    # 4-bit codes of Gaussian weights, two to a byte: byte values are drawn from a table of Gaussian pairs
    pairs = torch.clamp(torch.round(8 + 2.6 * torch.randn((65536, 2), generator=g, device="cuda")), 0, 15).to(torch.uint8)
    table = pairs[:, 0] | (pairs[:, 1] << 4)
    s["codes"] = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    for e in range(E):
        s["codes"][e] = table[torch.randint(0, 65536, (N, K // 2), generator=g, device="cuda", dtype=torch.int32)]
    s["scales"] = (torch.rand((E, N, G), generator=g, device="cuda") * 0.006 + 0.004).to(t)
    s["zeros"] = torch.randint(5, 11, (E, N, G), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    s["x"] = gauss(T, K)
    s["out"] = torch.zeros((T * k, N // 2 if case["swiglu"] else N), dtype=t, device="cuda")
    s["expert_off"], _, s["row_pair"] = _sorted(_routing(g, T, E, k, 0.0)[0], E)
    return s


# ---------------------------------------------------------------- the operators

RESIDUAL_SCALE, BRANCH_SCALE = 1.0, 0.7


def _own(s):
    from paper_2608_14385_b200 import binding
    c, op = s["case"], s["case"]["op"]
    kind = {"channel": binding.GATE_CHANNEL, "token": binding.GATE_TOKEN, "full": binding.GATE_FULL}.get(c.get("gate"))
    if op == "tokens":
        off, pair_row, row_pair = binding.sort_pairs(s["idx"], c["experts"])
        rows = binding.dispatch(s["x"], pair_row, rows=s["rows"])
        return off, pair_row, row_pair, rows, binding.combine(s["y"], pair_row, s["w"])
    if op == "tokens_backward":
        dy, dw = binding.combine_backward(s["dout"], s["y"], s["pair_row"], s["w"], drows=s["rows"])
        return dy, dw, binding.dispatch_backward(s["drows"], s["pair_row"])
    if op == "norms":
        h = binding.norm(s["x"], s["w_pre"], EPS)
        out, u = binding.norm_residual(s["x"], s["y"], s["w_post"], EPS, gate=s["gate"], residual_scale=RESIDUAL_SCALE,
                                       branch_scale=BRANCH_SCALE, next_weight=s["w_next"], gate_kind=kind)
        return h, out, u
    if op == "norms_backward":
        dx, dy, dgate, dw, dnext = binding.norm_residual_backward(
            s["x"], s["y"], s["w_post"], EPS, s["dout"], gate=s["gate"], residual_scale=RESIDUAL_SCALE,
            branch_scale=BRANCH_SCALE, next_weight=s["w_next"], du=s["du"], gate_kind=kind)
        dx_pre, dpre = binding.norm_backward(s["x"], s["w_pre"], EPS, s["dh"], dadd=s["dout"])
        return [dx, dy, dw, dnext, dx_pre, dpre] + ([] if dgate is None else [dgate])
    return binding.quant_product(s["codes"], s["scales"], s["x"], c["group"], zeros=s["zeros"],
                                 expert_off=s["expert_off"], row_pair=s["row_pair"], pairs_per_token=c["top_k"],
                                 swiglu=c["swiglu"], out=s["out"])


def _rms(v):
    return torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)


def _norm_grad(v, d):
    """Gradient through v * rms(v), for the gradient d of the result."""
    r = _rms(v)
    return r * d - v * (r * r * r) * (d * v).mean(dim=1, keepdim=True)


def _block(s):
    """The sum after the block in 32 bits, and what it is made of."""
    x, y, w = s["x"].float(), s["y"].float(), s["w_post"].float()
    kind = s["case"]["gate"]
    gate = 1.0 if kind == "none" else s["gate"].float()
    gate = gate[:, None] if kind == "token" else gate
    normed = y * _rms(y)
    return x, y, w, gate, normed, RESIDUAL_SCALE * x + BRANCH_SCALE * gate * (normed * w)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    t = TYPES[c["type"]]
    if op == "tokens":
        off, pair_row, row_pair = _sorted(s["idx"], c["experts"])
        token = row_pair.long().clamp(min=0) // c["top_k"]
        rows = torch.where((row_pair >= 0)[:, None], s["x"][token], s["rows"])
        return off, pair_row, row_pair, rows, _back(s["y"], pair_row, s["w"]).to(t)
    if op == "tokens_backward":
        at = s["pair_row"].long().reshape(-1)
        ok = at >= 0
        k, P = c["top_k"], at.numel()
        row_pair = torch.full((P + 1,), -1, dtype=torch.long, device=at.device)
        row_pair[torch.where(ok, at, torch.full_like(at, P))] = torch.arange(P, device=at.device)
        row_pair = row_pair[:P]
        token = row_pair.clamp(min=0) // k
        dy = s["dout"][token].float() * s["w"].reshape(-1)[row_pair.clamp(min=0)][:, None]
        dy = torch.where((row_pair >= 0)[:, None], dy.to(t), s["rows"])
        rows = s["y"][s["pair_row"].long().clamp(min=0)].float()
        dw = (rows * s["dout"].float()[:, None, :]).sum(dim=2)
        dw = torch.where(s["pair_row"] >= 0, dw, torch.zeros_like(dw))
        return dy, dw, _back(s["drows"], s["pair_row"], torch.ones_like(s["w"])).to(t)
    if op == "norms":
        x, _, _, _, _, out = _block(s)
        return (x * _rms(x) * s["w_pre"].float()).to(t), out.to(t), (out * _rms(out) * s["w_next"].float()).to(t)
    if op == "norms_backward":
        x, y, w, gate, normed, out = _block(s)
        du, dh = s["du"].float(), s["dh"].float()
        d = s["dout"].float() + _norm_grad(out, du * s["w_next"].float())
        dv = BRANCH_SCALE * gate * d
        dgate = BRANCH_SCALE * d * (normed * w)
        dx_pre = s["dout"].float() + _norm_grad(x, dh * s["w_pre"].float())
        got = [(RESIDUAL_SCALE * d).to(t), _norm_grad(y, dv * w).to(t), (dv * normed).sum(dim=0),
               (du * out * _rms(out)).sum(dim=0), dx_pre.to(t), (dh * x * _rms(x)).sum(dim=0)]
        kind = c["gate"]
        return got + ([] if kind == "none" else [dgate.sum(dim=0)] if kind == "channel" else [dgate.sum(dim=1)] if kind == "token"
                      else [dgate.to(t)])
    R = s["row_pair"].numel()
    row = torch.arange(R, device="cuda", dtype=torch.int32)
    expert = torch.searchsorted(s["expert_off"], row, right=True) - 1
    filled = row < s["expert_off"][-1]
    expert = expert.clamp(max=c["experts"] - 1)
    codes = s["codes"][expert]
    w = torch.stack([codes & 15, codes >> 4], dim=3).view(R, c["rows"], c["cols"]).float()
    spread = torch.arange(c["cols"], device="cuda") // c["group"]
    w.sub_(8.0 if s["zeros"] is None else s["zeros"][expert][:, :, spread])
    w.mul_(s["scales"][expert][:, :, spread])
    v = torch.bmm(w, s["x"][s["row_pair"].long().clamp(min=0) // c["top_k"]].float()[:, :, None])[:, :, 0]
    if c["swiglu"]:
        gate, up = v.chunk(2, dim=1)
        v = gate / (1.0 + torch.exp(-gate)) * up
    return torch.where(filled[:, None], v.to(t), s["out"])


def _back(rows, pair_row, w):
    """Weighted sum of every token's rows, in 32 bits."""
    taken = rows[pair_row.long().clamp(min=0)].float() * w[:, :, None]
    return torch.where((pair_row >= 0)[:, :, None], taken, torch.zeros_like(taken)).sum(dim=1)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 2 if case["type"] == "bf16" else 4
    op = case["op"]
    if op in ("tokens", "tokens_backward"):
        T, h, k, n = case["tokens"], case["hidden"], case["top_k"], case["experts"]
        P, kept = T * k, T * k * (1.0 - case["drop"])
        if op == "tokens":  # indices in, three lists out; x in, rows out; rows and weights in, out
            return {"bytes": 12 * P + 4 * (n + 1) + (2 * T + 2 * kept) * h * size + 4 * P, "flops": 2.0 * kept * h}
        return {"bytes": 12 * P + (2 * T + 3 * kept) * h * size, "flops": 4.0 * kept * h}
    if op in ("norms", "norms_backward"):
        T, h = case["tokens"], case["hidden"]
        full = 1 if case["gate"] == "full" else 0
        if op == "norms":  # x in, h out; y (and the gate) in, out and u out
            return {"bytes": (5 + full) * T * h * size, "flops": 14.0 * T * h}
        # x, y, dout, du, dh (and the gate) in, two dx and dy (and dgate) out
        return {"bytes": (8 + 2 * full) * T * h * size, "flops": 40.0 * T * h}
    E, N, K, T, k = case["experts"], case["rows"], case["cols"], case["tokens"], case["top_k"]
    active = E * (1.0 - (1.0 - k / E) ** T)
    G = -(-K // case["group"])
    weights = active * N * (K // 2 + G * (size + (1 if case["zeros"] else 0)))
    return {"bytes": weights + T * K * size + T * k * (N // 2 if case["swiglu"] else N) * size, "flops": 2.0 * T * k * N * K}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    """What run returns, from each operator's definition in 64 bits: expert by expert, slot by slot, and the gradients
    of the norms by differentiating their definition."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("tokens", "tokens_backward"):
        T, k, h, n = case["tokens"], case["top_k"], case["hidden"], case["experts"]
        flat = s["idx"].reshape(-1).cpu().tolist()
        lists = [[] for _ in range(n)]
        for p, e in enumerate(flat):
            if 0 <= e < n:
                lists[e].append(p)
        off, row_pair = [0], []
        for pairs in lists:
            row_pair += pairs
            off.append(len(row_pair))
        pair_row = [-1] * (T * k)
        for r, p in enumerate(row_pair):
            pair_row[p] = r
        order = torch.tensor(row_pair, dtype=torch.long, device="cuda")
        R = len(row_pair)
        w = s["w"].double()
        back = torch.zeros((T, h), dtype=torch.float64, device="cuda")
        rows = s["rows"].double()
        if op == "tokens":
            rows[:R] = s["x"].double()[order // k]
            scaled = s["y"][:R].double() * w.reshape(-1)[order][:, None]
            back.index_add_(0, order // k, scaled)
            ints = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (off, pair_row, row_pair + [-1] * (T * k - R))]
            return ints[0], ints[1].view(T, k), ints[2], rows, back
        dout = s["dout"].double()[order // k]
        rows[:R] = dout * w.reshape(-1)[order][:, None]
        dw = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        dw[order] = torch.linalg.vecdot(dout, s["y"][:R].double())
        back.index_add_(0, order // k, s["drows"][:R].double())
        return rows, dw.view(T, k), back
    if op in ("norms", "norms_backward"):
        leaf = {n: s[n].double().requires_grad_(op == "norms_backward") for n in ("x", "y", "w_pre", "w_post", "w_next")}
        gate = None if s["gate"] is None else s["gate"].double().requires_grad_(op == "norms_backward")
        over = {"none": None, "channel": (1, -1), "token": (-1, 1), "full": s["x"].shape}[case["gate"]]

        def unit(v):
            return v / torch.sqrt(v.pow(2).sum(dim=1, keepdim=True) / v.shape[1] + EPS)

        branch = unit(leaf["y"]) * leaf["w_post"]
        branch = branch if gate is None else branch * gate.reshape(over)
        out = RESIDUAL_SCALE * leaf["x"] + BRANCH_SCALE * branch
        u = unit(out) * leaf["w_next"]
        h = unit(leaf["x"]) * leaf["w_pre"]
        if op == "norms":
            return h, out, u
        after = [leaf["x"], leaf["y"], leaf["w_post"], leaf["w_next"]] + ([] if gate is None else [gate])
        got = torch.autograd.grad([out, u], after, [s["dout"].double(), s["du"].double()])
        # before the block the stream's own gradient joins that of the norm
        before = torch.autograd.grad([h, 1.0 * leaf["x"]], [leaf["x"], leaf["w_pre"]], [s["dh"].double(), s["dout"].double()])
        return list(got[:4]) + list(before) + list(got[4:])
    E, N, K = case["experts"], case["rows"], case["cols"]
    off, pairs = s["expert_off"].cpu().tolist(), s["row_pair"].long()
    out = s["out"].double()
    for e in range(E):
        if off[e] == off[e + 1]:
            continue
        w = torch.empty((N, K), dtype=torch.float64, device="cuda")
        w[:, 0::2] = torch.remainder(s["codes"][e], 16).double()
        w[:, 1::2] = torch.div(s["codes"][e], 16, rounding_mode="floor").double()
        z = torch.full_like(s["scales"][e], 8.0).double() if s["zeros"] is None else s["zeros"][e].double()
        w -= torch.repeat_interleave(z, case["group"], dim=1)[:, :K]
        w *= torch.repeat_interleave(s["scales"][e].double(), case["group"], dim=1)[:, :K]
        v = s["x"].double()[pairs[off[e]:off[e + 1]] // case["top_k"]] @ w.T
        out[off[e]:off[e + 1]] = torch.sigmoid(v[:, :N // 2]) * v[:, :N // 2] * v[:, N // 2:] if case["swiglu"] else v
    return out
