"""Refusals of the router, the experts' products and combine's gradient, on the host: every documented argument
error is returned before any HIP call. The pointers are fake addresses that nothing may dereference."""
import ctypes
import os

import pytest
import torch

from paper_2607_06202_amd import epl

OK, INVALID, ALIGN, CAPACITY, UNSUPPORTED = 0, 1, 2, 3, 5
P, ODD4, ODD2 = 0x10000, 0x10008, 0x10002  # 16-byte aligned; not 16; not 4
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(epl.LIB_PATH):
        from paper_2607_06202_amd import _build
        _build.build()
    return epl.lib()


def buffers(**kw):
    f = {n: P for n, _ in epl.LayoutBuffers._fields_}
    f.update(kw)
    return epl.LayoutBuffers(**f)


CFG = epl.config(2, 8, 2, 128, 4)  # T = 8, T*k = 16
BAD_CFG = epl.config(3, 8, 2, 128, 4)


def opts(logits=0, score=0, normalize=1, scale=1.0):
    return epl.RouteOpts(logits, score, normalize, scale)


def route(lib, cfg=CFG, o=None, logits=P, bias=None, idx=P, w=P):
    return lib.epl_route(ctypes.byref(cfg), ctypes.byref(o or opts()), logits, bias, idx, w, None)


def test_route_refusals(lib):
    assert route(lib, cfg=BAD_CFG) == INVALID
    for bad in (opts(logits=2), opts(score=2), opts(normalize=2), opts(scale=NAN), opts(scale=float("inf"))):
        assert route(lib, o=bad) == INVALID
    assert lib.epl_route(ctypes.byref(CFG), None, P, None, P, P, None) == INVALID
    assert route(lib, logits=None) == route(lib, idx=None) == route(lib, w=None) == INVALID
    assert route(lib, logits=ODD2) == route(lib, idx=ODD2) == route(lib, w=ODD2) == route(lib, bias=ODD2) == ALIGN
    assert route(lib, o=opts(logits=1), logits=P + 1) == ALIGN
    assert route(lib, cfg=epl.config(2, 8, 2, 128, 0), logits=None, idx=None, w=None) == OK  # no tokens, no launch


def test_route_backward_refusals(lib):
    def call(o=None, logits=P, idx=P, dw=P, dl=2 * P):
        return lib.epl_route_backward(ctypes.byref(CFG), ctypes.byref(o or opts()), logits, idx, dw, dl, None)

    assert call(logits=None) == call(idx=None) == call(dw=None) == call(dl=None) == INVALID
    assert call(dl=P) == INVALID  # dlogits is logits
    assert call(dl=ODD2) == call(dw=ODD2) == ALIGN
    assert call(o=opts(score=-1)) == INVALID


def gated(lib, cfg=CFG, inner=64, act=1, stride=0, recv=P, rs=P, rows=16, L=None, wg=P, wu=P, gs=P, us=P, h=P, pre=P):
    g = epl.Gated(inner, act, stride)
    bufs = L or buffers()
    return lib.epl_experts_gated(ctypes.byref(cfg), ctypes.byref(g), recv, rs, rows, ctypes.byref(bufs), wg, wu, gs,
                                 us, h, pre, None)


def test_gated_refusals(lib):
    assert gated(lib, cfg=BAD_CFG) == INVALID
    for inner in (0, 4, 12, -8, (1 << 20) + 8):
        assert gated(lib, inner=inner) == INVALID, inner
    assert gated(lib, act=4) == gated(lib, act=-1) == INVALID
    assert gated(lib, stride=64 * 128 - 8) == gated(lib, stride=64 * 128 + 4) == gated(lib, stride=-8) == INVALID
    assert gated(lib, stride=1 << 62) == INVALID
    assert gated(lib, rows=15) == CAPACITY
    assert gated(lib, L=buffers(expert_off=None)) == INVALID
    assert gated(lib, L=buffers(expert_off=ODD2)) == ALIGN
    for name in ("recv", "wg", "wu", "h"):
        assert gated(lib, **{name: None}) == INVALID, name
        assert gated(lib, **{name: ODD4}) == ALIGN, name
    assert gated(lib, pre=ODD4) == ALIGN
    f8 = epl.config(2, 8, 2, 128, 4, "fp8")
    for name in ("rs", "gs", "us"):
        assert gated(lib, cfg=f8, **{name: None}) == INVALID, name
        assert gated(lib, cfg=f8, **{name: ODD2}) == ALIGN, name
    assert gated(lib, cfg=f8, stride=64 * 128 + 8) == INVALID  # E4M3 matrices in 16-byte pieces
    assert gated(lib, cfg=epl.config(2, 8, 2, 136, 4, "fp8")) == UNSUPPORTED
    assert gated(lib, cfg=epl.config(2, 8, 2, 128, 0), recv=None, h=None, wg=None, wu=None, rows=0) == OK


def test_gated_backward_refusals(lib):
    names = ["dh", "pre", "recv", "wg", "wu", "dpre", "drecv", "dwg", "dwu"]

    def call(cfg=CFG, rows=16, **kw):
        v = dict({n: P for n in names}, drecv=2 * P, **kw) if "drecv" not in kw else dict({n: P for n in names}, **kw)
        g, L = epl.Gated(64, 1, 0), buffers()
        return lib.epl_experts_gated_backward(ctypes.byref(cfg), ctypes.byref(g), v["dh"], v["pre"], v["recv"], rows,
                                              ctypes.byref(L), v["wg"], v["wu"], v["dpre"], v["drecv"], v["dwg"],
                                              v["dwu"], None)

    for n in names:
        assert call(**{n: None}) == INVALID, n
        assert call(**{n: ODD4}) == ALIGN, n
    assert call(drecv=P) == INVALID
    assert call(rows=15) == CAPACITY
    assert call(cfg=epl.config(2, 8, 2, 128, 4, "fp8")) == UNSUPPORTED


def lin(K=64, N=32, ip=0, op=0, rp=0, act=0, payload=0, stride=0):
    return epl.Linear(K, N, ip, op, rp, act, payload, stride)


def linear(lib, l=None, a=P, asc=P, rows=16, w=P, wsc=P, bias=P, res=P, out=P, pre=P, L=None, cfg=CFG):
    bufs = L or buffers()
    return lib.epl_experts_linear(ctypes.byref(cfg), ctypes.byref(l or lin()), a, asc, rows, ctypes.byref(bufs), w,
                                  wsc, bias, res, out, pre, None)


def test_linear_refusals(lib):
    for bad in (lin(K=4), lin(N=12), lin(K=(1 << 20) + 8), lin(ip=56), lin(ip=68), lin(op=24), lin(op=36), lin(rp=24),
                lin(act=9), lin(stride=64), lin(stride=64 * 32 + 4), lin(ip=(1 << 20) + 64), lin(op=-64)):
        assert linear(lib, bad) == INVALID, (bad.in_features, bad.out_features, bad.in_pitch, bad.out_pitch)
    assert linear(lib, lin(payload=2)) == UNSUPPORTED
    assert linear(lib, lin(K=64, payload=1)) == UNSUPPORTED
    assert linear(lib, lin(K=128, ip=136, payload=1)) == INVALID  # E4M3 rows in 16-byte pieces
    assert linear(lib, lin(K=128, payload=1), asc=None) == INVALID
    assert linear(lib, lin(K=128, payload=1), wsc=ODD2) == ALIGN
    assert linear(lib, rows=15) == CAPACITY
    assert linear(lib, cfg=BAD_CFG) == INVALID
    for name in ("a", "w", "out"):
        assert linear(lib, **{name: None}) == INVALID, name
    for name in ("a", "w", "out", "bias", "res", "pre"):
        assert linear(lib, **{name: ODD4}) == ALIGN, name
    assert linear(lib, cfg=epl.config(2, 8, 2, 128, 0), rows=0, a=None, w=None, out=None) == OK


def test_linear_backward_refusals(lib):
    def call(l=None, dy=P, pre=P, a=P, rows=16, w=P, dpre=P, da=2 * P, dw=P, db=P):
        L = buffers()
        return lib.epl_experts_linear_backward(ctypes.byref(CFG), ctypes.byref(l or lin(act=1)), dy, pre, a, rows,
                                               ctypes.byref(L), w, dpre, da, dw, db, None)

    for kw in (dict(dy=None), dict(pre=None), dict(a=None), dict(w=None), dict(dpre=None), dict(da=None), dict(dw=None),
               dict(da=P)):
        assert call(**kw) == INVALID, kw
    for n in ("dy", "pre", "a", "w", "dpre", "da", "dw", "db"):
        assert call(**{n: ODD4}) == ALIGN, n
    assert call(rows=15) == CAPACITY
    assert call(lin(K=128, payload=1)) == UNSUPPORTED


def test_combine_backward_refusals(lib):
    def call(cfg=CFG, dout=P, y=P, w=P, dy=P, rows=16, dw=P, L=None):
        bufs = L or buffers()
        return lib.epl_combine_backward(ctypes.byref(cfg), dout, y, w, ctypes.byref(bufs), dy, rows, dw, None)

    for n in ("dout", "y", "w", "dy", "dw"):
        assert call(**{n: None}) == INVALID, n
        assert call(**{n: ODD2}) == ALIGN, n
    assert call(rows=15) == CAPACITY
    assert call(cfg=BAD_CFG) == INVALID
    assert call(L=buffers(pair_row=None)) == INVALID


def test_buffers_that_would_race_are_refused(lib):
    """Outputs at the address of a buffer that other workgroups may still read, all other buffers apart."""
    def apart(*names):
        return {n: (i + 1) * P for i, n in enumerate(names)}

    one = ctypes.byref
    L = buffers(expert_off=64 * P, pair_row=65 * P)

    def gated_(**same):
        v = apart("recv", "wg", "wu", "h", "pre")
        v.update({a: v[b] for a, b in same.items()})
        return lib.epl_experts_gated(one(CFG), one(epl.Gated(64, 1, 0)), v["recv"], None, 16, one(L), v["wg"], v["wu"],
                                     None, None, v["h"], v["pre"], None)

    def gated_back(**same):
        v = apart("dh", "pre", "recv", "wg", "wu", "dpre", "drecv", "dwg", "dwu")
        v.update({a: v[b] for a, b in same.items()})
        return lib.epl_experts_gated_backward(one(CFG), one(epl.Gated(64, 1, 0)), v["dh"], v["pre"], v["recv"], 16,
                                              one(L), v["wg"], v["wu"], v["dpre"], v["drecv"], v["dwg"], v["dwu"], None)

    def linear_(l, **same):
        v = apart("a", "w", "bias", "res", "out", "pre")
        v.update({a: v[b] for a, b in same.items()})
        return lib.epl_experts_linear(one(CFG), one(l), v["a"], None, 16, one(L), v["w"], None, v["bias"], v["res"],
                                      v["out"], v["pre"], None)

    def linear_back(l, **same):
        v = apart("dy", "pre", "a", "w", "dpre", "da", "dw", "db")
        v.update({a: v[b] for a, b in same.items()})
        return lib.epl_experts_linear_backward(one(CFG), one(l), v["dy"], v["pre"], v["a"], 16, one(L), v["w"],
                                               v["dpre"], v["da"], v["dw"], v["db"], None)

    def combine_back(**same):
        v = apart("dout", "y", "w", "dy", "dw")
        v.update({a: v[b] for a, b in same.items()})
        return lib.epl_combine_backward(one(CFG), v["dout"], v["y"], v["w"], one(L), v["dy"], 16, v["dw"], None)

    for a, b in (("h", "recv"), ("h", "pre"), ("pre", "recv"), ("h", "wg"), ("pre", "wu")):
        assert gated_(**{a: b}) == INVALID, (a, b)
    for a, b in (("dpre", "dh"), ("dpre", "recv"), ("drecv", "recv"), ("drecv", "dpre"), ("drecv", "wu"), ("dwg", "dwu"),
                 ("dwu", "recv"), ("dwg", "dpre")):
        assert gated_back(**{a: b}) == INVALID, (a, b)
    for a, b in (("out", "a"), ("out", "w"), ("out", "pre"), ("pre", "a"), ("pre", "res")):
        assert linear_(lin(K=64, N=64), **{a: b}) == INVALID, (a, b)
    assert linear_(lin(rp=40), out="res") == INVALID  # in place needs one pitch
    for a, b in (("dpre", "dy"), ("da", "a"), ("da", "dpre"), ("da", "w"), ("dw", "a"), ("db", "dw"), ("db", "dpre")):
        assert linear_back(lin(act=1), **{a: b}) == INVALID, (a, b)
    for a, b in (("da", "dy"), ("dw", "dy"), ("db", "dy")):
        assert linear_back(lin(), **{a: b}) == INVALID, (a, b)
    for a, b in (("dy", "dout"), ("dw", "w")):
        assert combine_back(**{a: b}) == INVALID, (a, b)


def test_binding_refuses_cpu_tensors_and_wrong_names():
    l = torch.zeros(8, 8)
    with pytest.raises(ValueError):
        epl.route(CFG, l)
    with pytest.raises(ValueError):
        epl.experts_gated(CFG, torch.zeros(16, 128, dtype=torch.bfloat16), None, l, l)
    with pytest.raises(ValueError):
        epl.experts_linear(CFG, torch.zeros(16, 128, dtype=torch.bfloat16), None, l)
    with pytest.raises(ValueError):
        epl._one_of(epl.ACTIVATION, "swish", "activation")
