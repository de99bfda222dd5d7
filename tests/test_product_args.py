"""Argument errors of the feed-forward blocks, the products and the 8-bit norms, found on the host before any CUDA call (no GPU needed)."""
import pytest
import torch

from paper_2608_14385_b200 import binding

INVALID, UNSUPPORTED, BATCH = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_BATCH
# addresses that are never read
A, B, D, E, F, G, H, W = (0x10000 * i for i in range(1, 9))


def _call(name, good, **change):
    args = dict(good, **change)
    return getattr(binding.lib(), name)(*[args[k] for k in good])


def _refused(name, good, cases):
    for change, want in cases:
        assert _call(name, good, **change) == want, change


def test_ffn():
    need = binding.lib().deamoe_ffn_workspace(4, 100, 64, 32, 0)
    assert need >= 100 * 32 * 2 and binding.lib().deamoe_ffn_workspace(4, 0, 64, 32, 0) == 0
    good = dict(s=None, x=A, xs=64, wgu=B, wd=D, off=E, E=4, R=100, h=64, f=32, out=F, os=64, ws=W, size=need)
    shared = [(dict(x=None), INVALID), (dict(x=A + 2), INVALID), (dict(xs=56), INVALID), (dict(xs=68), INVALID), (dict(wgu=None), INVALID),
              (dict(wgu=B + 8), INVALID), (dict(wd=None), INVALID), (dict(wd=D + 2), INVALID), (dict(off=None), INVALID),
              (dict(off=E + 2), INVALID), (dict(E=0), INVALID), (dict(E=2049), UNSUPPORTED), (dict(R=-1), BATCH), (dict(h=0), INVALID),
              (dict(h=60, xs=64), UNSUPPORTED), (dict(f=33), UNSUPPORTED), (dict(h=2 ** 20 + 8, xs=2 ** 21), UNSUPPORTED),
              (dict(f=2 ** 20 + 8), UNSUPPORTED), (dict(R=2 ** 31 - 1, h=2 ** 20, xs=2 ** 20), BATCH), (dict(ws=None), INVALID),
              (dict(ws=W + 8), INVALID)]
    _refused("deamoe_ffn", good, shared + [(dict(out=None), INVALID), (dict(out=A), INVALID), (dict(out=F + 8), INVALID), (dict(os=60), INVALID),
                                           (dict(os=66), INVALID), (dict(size=need - 1), INVALID), (dict(R=0), binding.OK)])
    need = binding.lib().deamoe_ffn_workspace(4, 100, 64, 32, 1)
    good = dict(s=None, x=A, xs=64, wgu=B, wd=D, dy=G, dys=64, off=E, E=4, R=100, h=64, f=32, dx=F, dxs=64, dwgu=H, dwd=0x90000, ws=W, size=need)
    _refused("deamoe_ffn_backward", good, shared + [
        (dict(dy=None), INVALID), (dict(dy=G + 2), INVALID), (dict(dys=63), INVALID), (dict(dx=None), INVALID), (dict(dx=A), INVALID),
        (dict(dx=G), INVALID), (dict(dxs=68), INVALID), (dict(dwgu=None), INVALID), (dict(dwd=None), INVALID), (dict(dwd=H), INVALID),
        (dict(dwgu=B), INVALID), (dict(dwd=D), INVALID), (dict(dwgu=H + 4), INVALID), (dict(size=need - 1), INVALID)])


def test_product():
    L = binding.lib()
    assert L.deamoe_product_workspace(1, 8, 7168, 7168, 0, 0) == 0 and L.deamoe_product_workspace(1, 64, 7168, 7168, 0, 0) > 0
    assert L.deamoe_product_workspace(1, 8192, 7168, 7168, 0, 0) == 0 and L.deamoe_product_workspace(1, 0, 8, 8, 1, 1) == 0
    good = dict(s=None, dt=1, x=A, xs=64, sx=None, T=8, w=B, sw=None, N=24, K=64, bdt=0, bias=D, act=1, res=E, rs=24, out=F, os=24, ws=None,
                size=0)
    shared = [(dict(x=None), INVALID), (dict(x=A + 8), INVALID), (dict(xs=56), INVALID), (dict(xs=68), INVALID), (dict(w=None), INVALID),
              (dict(w=B + 2), INVALID), (dict(T=-1), BATCH), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(K=60), UNSUPPORTED),
              (dict(K=2 ** 20 + 64, xs=2 ** 21), UNSUPPORTED), (dict(N=2 ** 20 + 8, os=2 ** 21, rs=2 ** 21), UNSUPPORTED), (dict(bdt=2), INVALID),
              (dict(bias=D + 2), INVALID), (dict(act=3), INVALID), (dict(act=-1), INVALID), (dict(dt=0), INVALID), (dict(dt=3), INVALID)]
    _refused("deamoe_product", good, shared + [
        (dict(out=None), INVALID), (dict(out=F + 1), INVALID), (dict(os=23), INVALID), (dict(out=A), INVALID), (dict(out=B), INVALID),
        (dict(res=E + 1), INVALID), (dict(rs=23), INVALID), (dict(res=F, rs=32), INVALID), (dict(sx=G), INVALID), (dict(sw=G), INVALID),
        (dict(dt=2), INVALID), (dict(dt=2, sx=G, sw=H, K=72, xs=80), UNSUPPORTED), (dict(dt=2, sx=G, sw=H, xs=72), INVALID),
        (dict(dt=2, sx=G + 2, sw=H), INVALID), (dict(T=2 ** 31 - 1, N=2 ** 20, os=2 ** 20, rs=2 ** 20), BATCH),
        (dict(T=64, K=7168, xs=7168, N=7168, os=7168, rs=7168), INVALID), (dict(T=0), binding.OK)])
    need = L.deamoe_product_workspace(1, 8, 24, 64, 1, 1)
    good = dict(s=None, dt=1, x=A, xs=64, T=8, w=B, N=24, K=64, bdt=0, bias=D, act=1, dout=E, ds=24, dx=F, dxs=64, dw=G, db=H, ws=W, size=need)
    _refused("deamoe_product_backward", good, [c for c in shared if "os" not in c[0]] + [
        (dict(dt=2), UNSUPPORTED), (dict(N=20, ds=24), UNSUPPORTED), (dict(dout=None), INVALID), (dict(dout=E + 2), INVALID), (dict(ds=16), INVALID),
        (dict(ds=28), INVALID), (dict(dx=None), INVALID), (dict(dx=A), INVALID), (dict(dx=E), INVALID), (dict(dx=B), INVALID),
        (dict(dxs=66), INVALID), (dict(dw=None), INVALID), (dict(dw=B), INVALID), (dict(dw=G + 2), INVALID), (dict(db=H + 2), INVALID),
        (dict(ws=None), INVALID), (dict(ws=W + 4), INVALID), (dict(size=need - 1), INVALID)])


def test_norm_quant():
    good = dict(s=None, dt=1, x=A, xs=64, T=4, h=64, norm=1, wdt=1, w=W, eps=1e-6, codes=B, cs=64, scale=D)
    _refused("deamoe_norm_quant", good, [
        (dict(dt=2), INVALID), (dict(wdt=2), INVALID), (dict(eps=-1.0), INVALID), (dict(norm=2), INVALID), (dict(x=None), INVALID),
        (dict(x=A + 1), INVALID), (dict(xs=63), INVALID), (dict(codes=None), INVALID), (dict(codes=A), INVALID), (dict(cs=63), INVALID),
        (dict(scale=None), INVALID), (dict(scale=D + 2), INVALID), (dict(w=W + 1), INVALID), (dict(T=-1), BATCH),
        (dict(h=2 ** 20 + 1, xs=2 ** 21, cs=2 ** 21), UNSUPPORTED), (dict(T=0), binding.OK)])
    good = dict(s=None, dt=1, x=A, xs=64, y=B, ys=64, T=4, h=64, norm=1, wdt=1, w=W, eps=1e-6, kind=1, gate=E, gs=0, a=1.0, b=1.0, out=D, os=64,
                wn=W, neps=1e-6, codes=F, cs=64, scale=G)
    _refused("deamoe_norm_residual_quant", good, [
        (dict(norm=0), INVALID), (dict(norm=2), INVALID), (dict(kind=0), INVALID), (dict(gate=None), INVALID), (dict(kind=3, gs=10), INVALID),
        (dict(y=None), INVALID), (dict(out=None), INVALID), (dict(out=B), INVALID), (dict(out=A, os=72), INVALID), (dict(codes=None), INVALID),
        (dict(codes=A), INVALID), (dict(codes=B), INVALID), (dict(codes=D), INVALID), (dict(cs=60), INVALID), (dict(scale=None), INVALID),
        (dict(scale=G + 1), INVALID), (dict(neps=float("nan")), INVALID), (dict(a=float("nan")), INVALID), (dict(T=-1), BATCH),
        (dict(T=0), binding.OK)])


def test_operator_status():
    assert binding.lib().deamoe_operator_status(None, None) == INVALID


class _NoCalls:
    """Stands in for the library: sizes of workspaces and the names of errors, no operator."""

    def __init__(self, real):
        self.deamoe_status_string = real.deamoe_status_string
        self.deamoe_ffn_workspace = self.deamoe_product_workspace = lambda *a: 0

    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def test_sizes_that_32_bits_cannot_hold_do_not_reach_the_library(monkeypatch):
    """ctypes passes the low 32 bits of what is larger."""
    stub = _NoCalls(binding.lib())
    monkeypatch.setattr(binding, "lib", lambda: stub)
    monkeypatch.setattr(binding, "_device", lambda: -1)          # CPU tensors pass for those of the current device
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    big = 2 ** 32
    one = torch.zeros((1, 1), dtype=torch.bfloat16)
    tall, long = one.expand(big + 8, 1), one.expand(1, big + 8)
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((8, 64), dtype=torch.bfloat16)
    wgu, wd = torch.zeros((1, 16, 64), dtype=torch.bfloat16), torch.zeros((1, 64, 8), dtype=torch.bfloat16)
    bad = [lambda: binding.product(tall, one, out=tall), lambda: binding.product(long, long, out=one), lambda: binding.product(one, tall, out=long),
           lambda: binding.product(x, w, act=big + 1), lambda: binding.product_backward(x, w, x[:, :8], act=big),
           lambda: binding.ffn(tall, wgu[:, :, :1], wd[:, :1], out=tall), lambda: binding.ffn(long, wgu, wd, out=long),
           lambda: binding.ffn(x, wgu.expand(big + 1, 16, 64), wd.expand(big + 1, 64, 8)),
           lambda: binding.ffn_backward(x, wgu, wd.expand(1, 64, 8)[:, :, :1].expand(1, 64, big + 8), x),
           lambda: binding.norm_quant(tall, None, 1e-6, codes=tall, scale=x[0]), lambda: binding.norm_quant(long, None, 1e-6, codes=long, scale=x[0])]
    for call in bad:
        with pytest.raises(binding.DeaMoEError) as e:
            call()
        assert e.value.status == INVALID


def test_workspaces_of_sums_over_more_than_a_stretch():
    """Contractions of more than 32768 values (8-bit: 65536) keep sums of their stretches: a CTA's half tile each, for what can overlap."""
    L, half = binding.lib(), 148 * 128 * 256 * 4
    assert L.deamoe_product_workspace(1, 32768, 8, 8, 0, 1) == 512 * 8 * 4
    assert L.deamoe_product_workspace(1, 32769, 8, 8, 0, 1) == -(-513 * 8 * 4 // 256) * 256 + 2 * half
    assert L.deamoe_product_workspace(1, 4096, 4096, 32768, 0, 0) == 0 and L.deamoe_product_workspace(1, 4096, 4096, 32776, 0, 0) == half
    assert L.deamoe_product_workspace(2, 4096, 4096, 65536, 0, 0) == 0 and L.deamoe_product_workspace(2, 4096, 4096, 65552, 0, 0) == half
    for R, h, f in ((32769, 8, 8), (20, 32776, 8), (20, 8, 16392)):
        v = [-(-R * f * n // 256) * 256 for n in (4, 4, 2)]
        assert L.deamoe_ffn_workspace(1, R, h, f, 1) == sum(v) + 3 * half
    assert L.deamoe_ffn_workspace(1, 32768, 8, 8, 1) == 32768 * 8 * 10
    need = L.deamoe_product_workspace(1, 40000, 8, 8, 0, 1)
    good = dict(s=None, dt=1, x=A, xs=8, T=40000, w=B, N=8, K=8, bdt=0, bias=D, act=0, dout=E, ds=8, dx=F, dxs=8, dw=G, db=H, ws=W, size=need)
    _refused("deamoe_product_backward", good, [(dict(size=need - 1), INVALID), (dict(ws=None), INVALID)])


@pytest.mark.parametrize("T", [2 ** 31 - 300, 2 ** 31 - 257, 2 ** 31 - 62, 2 ** 31 - 1])
def test_workspace_of_the_most_tokens(T):
    """Also for the few sizes beyond those that the call takes, so that it is the call that refuses them."""
    sums = 2 * 148 * 128 * 256 * 4
    for act, parts in ((0, -(-T // 64)), (1, 2 * -(-T // 64))):
        want = -(-parts * 8 * 4 // 256) * 256 + (0 if act == 0 else -(-T * 16 // 256) * 256) + sums
        assert binding.lib().deamoe_product_workspace(1, T, 8, 8, act, 1) == want
