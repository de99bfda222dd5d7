"""Argument errors of the operators around a layer, found on the host before any CUDA call (no GPU needed)."""
import pytest
import torch

from paper_2608_14385_b200 import binding

INVALID, UNSUPPORTED, BATCH = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_BATCH
A, B, D, E, W = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000   # addresses that are never read


def _call(name, good, **change):
    L = binding.lib()
    args = dict(good, **change)
    return getattr(L, name)(*[args[k] for k in good])


def test_sort():
    good = dict(s=None, idx=A, T=1000, k=8, n=64, off=B, pair=D, row=E, ws=W, size=1 << 30)
    L = binding.lib()
    assert L.deamoe_sort_workspace(192, 8, 64) == 0 and L.deamoe_sort_workspace(193, 8, 64) > 0
    for change, want in ((dict(n=0), INVALID), (dict(n=4096), UNSUPPORTED), (dict(k=0), INVALID), (dict(k=33), UNSUPPORTED),
                         (dict(T=-1), BATCH), (dict(T=2 ** 30, k=2), BATCH), (dict(idx=None), INVALID), (dict(off=None), INVALID),
                         (dict(pair=D + 2), INVALID), (dict(row=None), INVALID), (dict(ws=None), INVALID), (dict(size=64), INVALID)):
        assert _call("deamoe_sort_pairs", good, **change) == want, change


def test_rows():
    good = dict(s=None, dt=1, x=A, xs=64, pair=B, T=4, k=2, h=64, rows=D, rs=64, n=8)
    for change, want in ((dict(dt=2), INVALID), (dict(x=None), INVALID), (dict(x=A + 1), INVALID), (dict(xs=63), INVALID),
                         (dict(rs=63), INVALID), (dict(rows=A), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 31), INVALID),
                         (dict(h=0), INVALID), (dict(h=2 ** 20 + 1, xs=2 ** 21, rs=2 ** 21), UNSUPPORTED), (dict(T=-1), BATCH),
                         (dict(pair=None), INVALID), (dict(pair=B + 1), INVALID), (dict(T=0), binding.OK), (dict(n=0), binding.OK)):
        assert _call("deamoe_dispatch", good, **change) == want, change
    good = dict(s=None, dt=0, rows=A, rs=64, n=8, pair=B, w=W, T=4, k=2, h=64, out=D, os=64)
    for change, want in ((dict(w=None), INVALID), (dict(w=W + 2), INVALID), (dict(out=A), INVALID), (dict(out=None), INVALID),
                         (dict(rows=A + 2), INVALID), (dict(k=33), UNSUPPORTED), (dict(T=0), binding.OK)):
        assert _call("deamoe_combine", good, **change) == want, change
    good = dict(s=None, dt=0, dout=A, ds=64, rows=B, rs=64, n=8, pair=E, w=W, T=4, k=2, h=64, drows=D, drs=64, dw=0x60000)
    for change, want in ((dict(drows=None, dw=None), INVALID), (dict(rows=None), INVALID), (dict(drows=A), INVALID),
                         (dict(drows=B), INVALID), (dict(dw=0x60002), INVALID), (dict(ds=1), INVALID), (dict(T=0), binding.OK)):
        assert _call("deamoe_combine_backward", good, **change) == want, change


def test_norms():
    good = dict(s=None, dt=1, x=A, xs=64, T=4, h=64, wdt=1, w=W, eps=1e-6, out=B, os=64)
    for change, want in ((dict(dt=5), INVALID), (dict(wdt=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
                         (dict(x=A + 1), INVALID), (dict(out=A, os=72), INVALID), (dict(xs=60), INVALID), (dict(h=2 ** 21), UNSUPPORTED),
                         (dict(T=-4), BATCH), (dict(w=W + 1), INVALID), (dict(T=0), binding.OK)):
        assert _call("deamoe_norm", good, **change) == want, change
    need = binding.lib().deamoe_norm_workspace(4, 64)
    good = dict(s=None, dt=1, x=A, xs=64, T=4, h=64, wdt=1, w=W, eps=1e-6, du=B, us=64, add=None, adds=0, dx=D, dxs=64, dw=E,
                ws=0x60000, size=need)
    for change, want in ((dict(dw=None), INVALID), (dict(ws=None), INVALID), (dict(ws=0x60008), INVALID), (dict(size=need - 1), INVALID),
                         (dict(dx=A), INVALID), (dict(dx=B), INVALID), (dict(add=D, adds=72), INVALID), (dict(du=None), INVALID)):
        assert _call("deamoe_norm_backward", good, **change) == want, change
    good = dict(s=None, dt=1, x=A, xs=64, y=B, ys=64, T=4, h=64, norm=1, wdt=1, w=W, eps=1e-6, kind=1, gate=E, gs=0, a=1.0, b=1.0,
                out=D, os=64, wn=W, neps=1e-6, next=0x60000, ns=64)
    for change, want in ((dict(norm=0), INVALID), (dict(norm=2), INVALID), (dict(kind=0), INVALID), (dict(gate=None), INVALID),
                         (dict(kind=4), INVALID), (dict(kind=3, gs=10), INVALID), (dict(next=None), INVALID), (dict(next=A), INVALID),
                         (dict(out=B), INVALID), (dict(out=A, os=72), INVALID), (dict(neps=-1.0), INVALID), (dict(a=float("nan")), INVALID),
                         (dict(y=None), INVALID), (dict(T=0), binding.OK)):
        assert _call("deamoe_norm_residual", good, **change) == want, change
    good = dict(s=None, dt=1, x=A, xs=64, y=B, ys=64, T=4, h=64, norm=1, wdt=1, w=W, eps=1e-6, kind=1, gate=E, gs=0, a=1.0, b=1.0,
                dout=D, ds=64, wn=W, neps=1e-6, dn=0x60000, dns=64, dx=0x70000, dxs=64, dy=0x80000, dys=64, dg=0x90000, dgs=0,
                dw=0xa0000, dwn=0xb0000, ws=0xc0000, size=need)
    for change, want in ((dict(dw=None), INVALID), (dict(w=None), INVALID), (dict(dwn=None), INVALID), (dict(wn=None), INVALID),
                         (dict(dn=None), INVALID), (dict(dg=None), INVALID), (dict(kind=0, gate=None), INVALID), (dict(dx=A), INVALID),
                         (dict(dy=D), INVALID), (dict(dx=0x80000), INVALID), (dict(size=need - 4), INVALID), (dict(dg=0x90002), INVALID)):
        assert _call("deamoe_norm_residual_backward", good, **change) == want, change


def test_quant():
    need = binding.lib().deamoe_quant_workspace(1, 8, 256)
    good = dict(s=None, dt=1, codes=A, sdt=1, scales=B, zeros=None, E=8, N=64, K=256, group=64, x=D, xs=256, T=4, off=E, pair=W, ppt=2,
                R=8, swiglu=0, out=0x60000, os=64, ws=0x70000, size=need)
    for change, want in ((dict(dt=7), INVALID), (dict(sdt=7), INVALID), (dict(codes=A + 8), INVALID), (dict(codes=None), INVALID),
                         (dict(scales=B + 1), INVALID), (dict(group=48), INVALID), (dict(K=250), UNSUPPORTED), (dict(K=0), INVALID),
                         (dict(E=4096), UNSUPPORTED), (dict(off=None), INVALID), (dict(ppt=0), INVALID), (dict(R=-1), BATCH),
                         (dict(T=-1), BATCH), (dict(swiglu=2), INVALID), (dict(swiglu=1, N=63), UNSUPPORTED), (dict(out=D), INVALID),
                         (dict(os=63), INVALID), (dict(xs=255), INVALID), (dict(x=None), INVALID), (dict(pair=W + 1), INVALID),
                         (dict(R=0), binding.OK)):
        assert _call("deamoe_quant_product", good, **change) == want, change
    if need:
        assert _call("deamoe_quant_product", good, ws=None) == INVALID
        assert _call("deamoe_quant_product", good, size=need - 1) == INVALID


class _NoCalls:
    """Stands in for the library: sizes of workspaces and the names of errors, no operator."""

    def __init__(self, real):
        self.deamoe_status_string = real.deamoe_status_string
        self.deamoe_sort_workspace = self.deamoe_quant_workspace = self.deamoe_norm_workspace = lambda *a: 0

    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def test_sizes_that_32_bits_cannot_hold_do_not_reach_the_library(monkeypatch):
    """ctypes passes the low 32 bits of what is larger: a group of 2^32 + 32 would be one of 32 with one scale a row, -2^32 + 8
    experts would be 8 with room for none."""
    stub = _NoCalls(binding.lib())
    monkeypatch.setattr(binding, "lib", lambda: stub)
    monkeypatch.setattr(binding, "_device", lambda: -1)          # CPU tensors pass for those of the current device
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    big = 2 ** 32
    idx = torch.zeros((4, 2), dtype=torch.int32)
    codes, scales = torch.zeros((1, 16, 32), dtype=torch.uint8), torch.zeros((1, 16, 1))
    x = torch.zeros((4, 64))
    tall, long = torch.zeros((1, 1)).expand(big + 4, 1), torch.zeros((1, 1)).expand(1, big + 4)
    pairs = torch.zeros((1, 1), dtype=torch.int32)
    bad = [lambda: binding.sort_pairs(idx, big + 8), lambda: binding.sort_pairs(idx, 8 - big),
           lambda: binding.quant_product(codes, scales, x, big + 32), lambda: binding.quant_product(codes, scales, x, 32 - big),
           lambda: binding.quant_product(codes, torch.zeros((1, 16, 2)), x, 32, pairs_per_token=big + 1),
           lambda: binding.quant_product(codes.expand(big + 1, 16, 32), scales, x, 64),
           lambda: binding.norm(tall, None, 1e-6, out=tall), lambda: binding.norm(long, None, 1e-6, out=long),
           lambda: binding.dispatch(x[:1], pairs.expand(1, big + 1), rows=x)]
    for call in bad:
        with pytest.raises(binding.DeaMoEError) as e:
            call()
        assert e.value.status == INVALID
