"""Cases and plain forms of the products around a layer: the gated feed-forward block of experts over sorted rows, products
with bias, activation and residual (bf16, and 8-bit operands), and the norms that make 8-bit rows for them.

`own` selects what `run` does: False computes the operator from elementary torch operations in 32 bits, True calls the
library (paper_2608_14385_b200.binding).  Both take the state that `prepare` makes on the current CUDA device.

Operators, as a user calls them:
  ffn               rows in expert order through their experts' SwiGLU block
  ffn_backward      its gradients: rows, gate / up matrices, down matrices
  product           act(x W^T + bias) + residual, from bf16 or from e4m3 values with a scale a row
  product_backward  its gradients: x, W, bias (bf16)
  norm8             sum after a block and the next block's norm in e4m3 with a scale a row
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0

# Sizes: hidden 7168, ffn 2048, top-8 are the DeepSeek-V3 shape of synth.py (16 or 32 of its 256 experts: one GPU's share of a
# layer spread over 8 or 16), hidden 4096 its 7b shape.  Odd sizes are generic.


def listed():
    return [
        # one token through one expert (the always-on shared one): latency of a decode step
        dict(name="ffn one token", op="ffn", experts=1, hidden=7168, ffn=2048, tokens=1, top_k=1, drop=0.0),
        # 16 tokens of a decode step over a GPU's 32 experts: all their weights, a few rows each
        dict(name="ffn experts 16", op="ffn", experts=32, hidden=7168, ffn=2048, tokens=16, top_k=8, drop=0.0),
        # a prompt of 2048 tokens, top-8 of 16 experts: about 1000 rows an expert
        dict(name="ffn prompt 2048", op="ffn", experts=16, hidden=7168, ffn=2048, tokens=2048, top_k=8, drop=0.0),
        # the gradients of a training step of the same size
        dict(name="ffn gradient 2048", op="ffn_backward", experts=16, hidden=7168, ffn=2048, tokens=2048, top_k=8, drop=0.0),
        # a small model's training step: odd sizes, a tenth of the pairs dropped
        dict(name="ffn gradient ragged", op="ffn_backward", experts=10, hidden=1032, ffn=344, tokens=777, top_k=2, drop=0.1),
        # a projection of a decode step of 8 tokens with 8-bit operands
        dict(name="product 8-bit decode", op="product", type="e4m3", tokens=8, cols=7168, rows=7168, bias=True, act="none", residual=False),
        # the same projection for a prompt of 8192 tokens, back into the residual stream
        dict(name="product 8-bit prompt", op="product", type="e4m3", tokens=8192, cols=7168, rows=7168, bias=False, act="none", residual=True),
        # a prompt of 4096 tokens through a bf16 projection with bias and GeLU
        dict(name="product prompt 4096", op="product", type="bf16", tokens=4096, cols=7168, rows=4096, bias=True, act="gelu", residual=False),
        # the gradients of a training step of 4096 tokens, square matrix of the 7b shape
        dict(name="product gradient 4096", op="product_backward", type="bf16", tokens=4096, cols=4096, rows=4096, bias=True, act="silu"),
        # odd sizes, no activation: the plain linear layer of a small model
        dict(name="product gradient ragged", op="product_backward", type="bf16", tokens=1021, cols=1096, rows=520, bias=True, act="none"),
        # after the block of a decode step of 8 tokens
        dict(name="norm 8-bit decode", op="norm8", tokens=8, hidden=7168, normalise=True),
        # after the block of a prompt of 8192 tokens
        dict(name="norm 8-bit prompt", op="norm8", tokens=8192, hidden=7168, normalise=True),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "ffn_backward", "product", "product", "product_backward", "norm8"])
    if op.startswith("ffn"):
        hidden, ffn, experts = 8 * _between(rng, 8, 896), 8 * _between(rng, 8, 256), _between(rng, 1, 64)
        experts = max(1, min(experts, 16 * 7168 * 2048 // (hidden * ffn)))
        top_k = rng.randint(1, min(8, experts))
        most = 16384 * 7168 * 2048 // (hidden * ffn * top_k)
        return dict(op=op, experts=experts, hidden=hidden, ffn=ffn, tokens=_between(rng, 1, max(1, min(8192, most))), top_k=top_k,
                    drop=rng.choice([0.0, 0.0, 0.1, 0.6]))
    if op == "product":
        kind = rng.choice(["bf16", "e4m3"])
        cols = 16 * _between(rng, 4, 448)
        rows = rng.choice([_between(rng, 33, 7168), 64 * _between(rng, 1, 112)])
        most = 8192 * 7168 * 7168 // ((1 if kind == "e4m3" else 2) * cols * rows)
        return dict(op=op, type=kind, tokens=_between(rng, 1, min(8192, most)), cols=cols, rows=rows, bias=rng.random() < 0.5,
                    act=rng.choice(["none", "silu", "gelu"]), residual=rng.random() < 0.5)
    if op == "product_backward":
        cols, rows = 8 * _between(rng, 8, 512), 8 * _between(rng, 8, 512)
        return dict(op=op, type="bf16", tokens=_between(rng, 1, 4096), cols=cols, rows=rows, bias=rng.random() < 0.5,
                    act=rng.choice(["none", "silu", "gelu"]))
    hidden = rng.choice([_between(rng, 64, 7168), 256 * rng.randint(1, 28)])
    return dict(op=op, tokens=_between(rng, 1, min(16384, 8192 * 7168 // hidden)), hidden=hidden, normalise=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _offsets(g, tokens, experts, top_k, drop):
    """First row of every expert for the top-k of Gaussian logits, a share `drop` of the pairs left out: int32 [experts + 1]."""
    logits = torch.randn((tokens, experts), generator=g, device="cuda")
    idx = torch.topk(logits, top_k, dim=1).indices.reshape(-1)
    kept = (torch.rand(idx.shape, generator=g, device="cuda") >= drop).long()
    count = torch.zeros(experts, dtype=torch.long, device="cuda").scatter_add_(0, idx, kept)
    return torch.cat([torch.zeros_like(count[:1]), torch.cumsum(count, 0)]).to(torch.int32)


def _rows8(v):
    """Rows of v in e4m3 with a scale each."""
    scale = v.abs().amax(dim=1) / E4M3_MAX
    return (v / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def gauss(*shape, scale=1.0, mean=0.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(mean).to(dtype)

    op, s = case["op"], {"case": case}
    if op.startswith("ffn"):
        E, h, f, T, k = case["experts"], case["hidden"], case["ffn"], case["tokens"], case["top_k"]
        s["off"] = _offsets(g, T, E, k, case["drop"])
        s["x"] = gauss(T * k, h)
        s["w_gate_up"] = torch.empty((E, 2 * f, h), dtype=torch.bfloat16, device="cuda")
        s["w_down"] = torch.empty((E, h, f), dtype=torch.bfloat16, device="cuda")
        for e in range(E):
            s["w_gate_up"][e] = gauss(2 * f, h, scale=h ** -0.5)
            s["w_down"][e] = gauss(h, f, scale=f ** -0.5)
        s["out"] = torch.zeros((T * k, h), dtype=torch.bfloat16, device="cuda")
        if op == "ffn_backward":
            s["dout"] = gauss(T * k, h)
        return s
    if op == "norm8":
        T, h = case["tokens"], case["hidden"]
        s["x"], s["y"] = gauss(T, h, scale=2.0), gauss(T, h, scale=0.5)
        s["w_post"] = gauss(h, scale=0.2, mean=1.0) if case["normalise"] else None
        s["w_next"] = gauss(h, scale=0.2, mean=1.0)
        return s
    T, K, N = case["tokens"], case["cols"], case["rows"]
    s["x"], s["w"] = gauss(T, K), gauss(N, K, scale=K ** -0.5)
    s["x_scale"] = s["w_scale"] = None
    if case["type"] == "e4m3":
        s["x"], s["x_scale"] = _rows8(s["x"].float())
        s["w"], s["w_scale"] = _rows8(s["w"].float())
    s["bias"] = gauss(N, scale=0.3) if case["bias"] else None
    if op == "product":
        s["residual"] = gauss(T, N) if case["residual"] else None
    else:
        s["dout"] = gauss(T, N)
    return s


# ---------------------------------------------------------------- the operators

def _own(s):
    from paper_2608_14385_b200 import binding
    c, op = s["case"], s["case"]["op"]
    if op == "ffn":
        return binding.ffn(s["x"], s["w_gate_up"], s["w_down"], expert_off=s["off"], out=s["out"])
    if op == "ffn_backward":
        return binding.ffn_backward(s["x"], s["w_gate_up"], s["w_down"], s["dout"], expert_off=s["off"], dx=s["out"])
    if op == "norm8":
        return binding.norm_residual_quant(s["x"], s["y"], s["w_post"], EPS, normalise=c["normalise"], next_weight=s["w_next"])
    act = {"none": binding.SIGMA_NONE, "silu": binding.SIGMA_SILU, "gelu": binding.SIGMA_GELU}[c["act"]]
    if op == "product":
        return binding.product(s["x"], s["w"], bias=s["bias"], act=act, residual=s["residual"], x_scale=s["x_scale"],
                               weight_scale=s["w_scale"])
    dx, dw, db = binding.product_backward(s["x"], s["w"], s["dout"], bias=s["bias"], act=act)
    return [dx, dw] + ([] if db is None else [db])


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _places(s):
    """Experts' rows as one padded batch: index of every place's row, and which places hold one [experts, most]."""
    off = s["off"].long()
    count = off[1:] - off[:-1]
    most = max(1, int(count.max()))
    at = torch.arange(most, device="cuda")
    held = at[None, :] < count[:, None]
    return torch.where(held, off[:-1, None] + at[None, :], torch.zeros_like(off[:-1, None])), held


def _spread(v, at, held):
    return torch.where(held[:, :, None], v[at].float(), torch.zeros((), device="cuda"))


def _gather(v, at, held, into):
    """Rows of a padded batch back in their places; rows of no expert stay as they are in `into`."""
    out = into.clone()
    out[at[held]] = v[held].to(into.dtype)
    return out


def _act(name, z):
    if name == "silu":
        return z * _sigmoid(z)
    return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5))) if name == "gelu" else z


def _act_grad(name, z):
    if name == "silu":
        p = _sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op.startswith("ffn"):
        at, held = _places(s)
        x = _spread(s["x"], at, held)
        wgu, wd = s["w_gate_up"].float(), s["w_down"].float()
        g, u = torch.bmm(x, wgu.transpose(1, 2)).chunk(2, dim=2)
        p = _sigmoid(g)
        h = g * p * u
        if op == "ffn":
            return _gather(torch.bmm(h, wd.transpose(1, 2)), at, held, s["out"])
        dy = _spread(s["dout"], at, held)
        dh = torch.bmm(dy, wd)
        dwd = torch.bmm(dy.transpose(1, 2), h).to(torch.bfloat16)
        dgu = torch.cat([dh * u * p * (1.0 + g * (1.0 - p)), dh * g * p], dim=2)
        return (_gather(torch.bmm(dgu, wgu), at, held, s["out"]), torch.bmm(dgu.transpose(1, 2), x).to(torch.bfloat16), dwd)
    if op == "norm8":
        x, y = s["x"].float(), s["y"].float()
        if c["normalise"]:
            y = y * torch.rsqrt((y * y).mean(dim=1, keepdim=True) + EPS) * s["w_post"].float()
        out = x + y
        u = out * torch.rsqrt((out * out).mean(dim=1, keepdim=True) + EPS) * s["w_next"].float()
        scale = u.abs().amax(dim=1) / E4M3_MAX
        return out.to(torch.bfloat16), (u / scale[:, None]).to(torch.float8_e4m3fn), scale
    x, w = s["x"].float(), s["w"].float()
    if op == "product":
        z = torch.mm(x, w.t())
        if s["x_scale"] is not None:
            z = z * s["x_scale"][:, None] * s["w_scale"][None, :]
        z = z if s["bias"] is None else z + s["bias"].float()
        z = _act(c["act"], z)
        return (z if s["residual"] is None else z + s["residual"].float()).to(torch.bfloat16)
    dz = s["dout"].float()
    if c["act"] != "none":
        z = torch.mm(x, w.t())
        dz = dz * _act_grad(c["act"], z if s["bias"] is None else z + s["bias"].float())
    got = [torch.mm(dz, w).to(torch.bfloat16), torch.mm(dz.t(), x).to(torch.bfloat16)]
    return got + ([] if s["bias"] is None else [dz.sum(dim=0)])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op.startswith("ffn"):
        E, h, f, T, k = case["experts"], case["hidden"], case["ffn"], case["tokens"], case["top_k"]
        rows = T * k * (1.0 - case["drop"])
        active = E * (1.0 - (1.0 - k * (1.0 - case["drop"]) / E) ** T)
        if op == "ffn":
            return {"bytes": active * 6 * h * f + 4 * rows * h, "flops": 6.0 * rows * h * f}
        # gate and up once more, then one product for the gradient of h, two for x, three for the matrices
        return {"bytes": (active + E) * 6 * h * f + 6 * rows * h, "flops": 16.0 * rows * h * f}
    if op == "norm8":
        return {"bytes": 7 * case["tokens"] * case["hidden"] + 4 * case["tokens"], "flops": 14.0 * case["tokens"] * case["hidden"]}
    T, K, N = case["tokens"], case["cols"], case["rows"]
    size = 1 if case["type"] == "e4m3" else 2
    if op == "product":
        return {"bytes": size * (T + N) * K + (4 if case["residual"] else 2) * T * N, "flops": 2.0 * T * K * N}
    return {"bytes": 4 * (T + N) * K + 2 * T * N, "flops": (6.0 if case["act"] != "none" else 4.0) * T * K * N}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    """What run returns, from each operator's definition in 64 bits: expert by expert, and the gradients by differentiating
    the definition."""
    s = prepare(case, seed)
    op = case["op"]
    silu = torch.nn.functional.silu
    if op.startswith("ffn"):
        back = op == "ffn_backward"
        off = s["off"].cpu().tolist()
        out = s["out"].double()
        dgu = torch.zeros(s["w_gate_up"].shape, dtype=torch.float64, device="cuda") if back else None
        dwd = torch.zeros(s["w_down"].shape, dtype=torch.float64, device="cuda") if back else None
        for e in range(case["experts"]):
            lo, hi = off[e], off[e + 1]
            if lo == hi:
                continue
            leaf = [v.double().requires_grad_(back) for v in (s["x"][lo:hi], s["w_gate_up"][e], s["w_down"][e])]
            inner = torch.einsum("th,fh->tf", leaf[0], leaf[1])
            y = torch.einsum("tf,hf->th", silu(inner[:, :case["ffn"]]) * inner[:, case["ffn"]:], leaf[2])
            if back:
                out[lo:hi], dgu[e], dwd[e] = torch.autograd.grad(y, leaf, s["dout"][lo:hi].double())
            else:
                out[lo:hi] = y
        return (out, dgu, dwd) if back else out
    if op == "norm8":
        def unit(v):
            return v / torch.sqrt(v.pow(2).sum(dim=1, keepdim=True) / v.shape[1] + EPS)

        y = s["y"].double()
        out = s["x"].double() + (unit(y) * s["w_post"].double() if case["normalise"] else y)
        u = unit(out) * s["w_next"].double()
        scale = torch.linalg.vector_norm(u, ord=float("inf"), dim=1) / E4M3_MAX
        return out, u / scale.unsqueeze(1), scale
    back = op == "product_backward"
    act = {"none": lambda z: z, "silu": silu, "gelu": torch.nn.functional.gelu}[case["act"]]
    x, w = s["x"].double(), s["w"].double()
    if s["x_scale"] is not None:
        x, w = x * s["x_scale"].double().unsqueeze(1), w * s["w_scale"].double().unsqueeze(1)
    leaf = [x.requires_grad_(back), w.requires_grad_(back)]
    if s["bias"] is not None:
        leaf.append(s["bias"].double().requires_grad_(back))
    z = torch.einsum("tk,nk->tn", leaf[0], leaf[1])
    z = act(z + leaf[2] if len(leaf) == 3 else z)
    if back:
        return list(torch.autograd.grad(z, leaf, s["dout"].double()))
    return z if s["residual"] is None else z + s["residual"].double()
