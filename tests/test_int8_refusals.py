"""Refusals of dispatch with weights, its gradient, and the calls for int8 rows, on the host, each from a call that is right
in everything but one argument (its own status is then that of a launch where there is no device). The pointers are fake
addresses: on a machine with a GPU the unchanged calls would launch, so nothing runs there."""
import ctypes
import os

import pytest
import torch

from paper_2607_06202_amd import epl

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are fake, and a GPU would follow them")

OK, INVALID, ALIGN, CAPACITY, UNSUPPORTED, DEVICE = 0, 1, 2, 3, 5, 6
P = 0x10000
CFG = epl.config(2, 8, 2, 128, 4)  # T = 8, T*k = 16
WIDE = (1 << 20) + 16              # more features than EPL_MAX_HIDDEN
one = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(epl.LIB_PATH):
        from paper_2607_06202_amd import _build
        _build.build()
    return epl.lib()


def lin(K=128, N=64, ip=0, op=0, rp=0, act=1, payload=0, stride=0):
    return epl.Linear(K, N, ip, op, rp, act, payload, stride)


ARGS = {
    "weighted": lambda lib, v, L: lib.epl_dispatch_weighted(v["cfg"], v["x"], v["w"], L, v["recv"], v["rows"], None),
    "backward": lambda lib, v, L: lib.epl_dispatch_backward(v["cfg"], v["drecv"], v["rows"], v["x"], v["w"], L, v["dx"],
                                                            v["dw"], None),
    "int8": lambda lib, v, L: lib.epl_dispatch_int8(v["cfg"], v["x"], v["w"], L, v["recv"], v["rs"], v["rows"], None),
    "quantize": lambda lib, v, L: lib.epl_quantize_rows(v["cfg"], v["z"] and one(v["z"]), v["a"], v["rows"],
                                                        None if v.get("no_layout") else L, v["q"], v["qs"], None),
    "gated": lambda lib, v, L: lib.epl_experts_gated_int8(
        v["cfg"], v["g"] and one(v["g"]), v["recv"], v["rs"], v["rows"], L, v["wg"], v["wu"], v["gs"], v["us"], v["h"], None),
    "linear": lambda lib, v, L: lib.epl_experts_linear_int8(
        v["cfg"], v["l"] and one(v["l"]), v["a"], v["asc"], v["rows"], L, v["wt"], v["wsc"], v["bias"], v["res"], v["out"],
        None),
}


class Call:
    """An entry point with every buffer at an address of its own. call(name=value) changes that argument; a value that
    names another buffer stands for its address. vectors: 16-byte aligned buffers; words: 4-byte aligned."""

    def __init__(self, name, vectors, words, outputs, optional="", may=(), **config):
        self.name, self.vectors, self.words = name, vectors.split(), words.split()
        self.outputs, self.optional, self.may = outputs.split(), optional.split(), {frozenset(m) for m in may}
        self.buffers = self.vectors + self.words
        self.inputs = [n for n in self.buffers if n not in self.outputs]
        self.layout = {n: (64 + i) * P for i, (n, _) in enumerate(epl.LayoutBuffers._fields_)}
        self.at = {n: (i + 1) * P for i, n in enumerate(self.buffers) if n not in self.layout}
        self.config = config

    def __call__(self, lib, **kw):
        v = dict(dict(cfg=CFG, rows=16, **self.config), **self.at, **self.layout)
        v.update({n: v[x] if isinstance(x, str) else x for n, x in kw.items()})
        L = epl.LayoutBuffers(*[v[n] for n, _ in epl.LayoutBuffers._fields_])
        v["cfg"] = None if v["cfg"] is None else one(v["cfg"])
        return ARGS[self.name](lib, v, None if v.get("null_layout") else one(L))


CALLS = {
    "weighted": Call("weighted", "x recv", "w pair_row", "recv"),
    "backward": Call("backward", "drecv x dx", "w dw pair_row", "dx dw", may=[("dx", "x")]),
    "int8": Call("int8", "x recv", "w rs pair_row", "recv rs", "w"),
    "quantize": Call("quantize", "a q", "qs expert_off", "q qs", z=epl.Quantize(128, 0, 0)),
    "gated": Call("gated", "recv wg wu h", "rs gs us expert_off", "h", g=epl.Gated(64, 1, 0)),
    "linear": Call("linear", "a wt bias res out", "asc wsc expert_off", "out", "bias res", may=[("out", "res")], l=lin()),
}


@pytest.mark.parametrize("name", CALLS)
def test_an_output_at_the_address_of_another_buffer(lib, name):
    call = CALLS[name]
    assert call(lib) == DEVICE
    for i, o in enumerate(call.outputs):
        for other in call.inputs + call.outputs[:i]:
            want = DEVICE if frozenset((o, other)) in call.may else INVALID
            assert call(lib, **{o: other}) == want, (o, other)


@pytest.mark.parametrize("name", CALLS)
def test_missing_and_misaligned_buffers(lib, name):
    call = CALLS[name]
    at = dict(call.layout, **call.at)
    for n in call.buffers:
        assert call(lib, **{n: None}) == (DEVICE if n in call.optional else INVALID), n
        assert call(lib, **{n: at[n] + (2 if n in call.words else 8)}) == ALIGN, n
    for n in call.layout:
        if n not in call.buffers:
            assert call(lib, **{n: None}) == call(lib, **{n: at[n] + 1}) == DEVICE, n
    assert call(lib, null_layout=True) == (DEVICE if name == "quantize" else INVALID)


@pytest.mark.parametrize("name", CALLS)
def test_bad_configs_and_row_counts(lib, name):
    call = CALLS[name]
    for bad in (None, epl.config(3, 8, 2, 128, 4), epl.config(2, 8, 0, 128, 4), epl.config(2, 8, 2, 124, 4),
                epl.config(2, 8, 2, 128, -1), epl.config(2, 8, 2, 128, 4, "bf16", 100)):
        assert call(lib, cfg=bad) == INVALID
    for rows in (15, 0, -1):
        assert call(lib, rows=rows) == CAPACITY
    assert call(lib, rows=17) == DEVICE
    assert call(lib, cfg=epl.config(2, 8, 2, 128, 4, "fp8")) == DEVICE  # the payload is not looked at
    wide = epl.config(2, 8, 2, 136, 4)  # a multiple of 8 alone
    if name in ("int8", "gated"):
        assert call(lib, cfg=wide) == UNSUPPORTED
    else:
        assert call(lib, cfg=wide) == DEVICE


@pytest.mark.parametrize("name", CALLS)
def test_without_tokens_nothing_is_needed(lib, name):
    call = CALLS[name]
    none = {n: None for n in call.at}
    assert call(lib, cfg=epl.config(2, 8, 2, 128, 0), rows=0, **none) == OK


def test_quantize_fields(lib):
    call = CALLS["quantize"]
    z = epl.Quantize
    for bad in (None, z(0, 0, 0), z(-16, 0, 0), z(12, 0, 0), z(WIDE, 0, 0), z(128, 120, 0), z(128, 132, 0), z(128, 0, 120),
                z(128, 0, 136), z(128, -128, 0), z(128, 0, WIDE)):
        assert call(lib, z=bad) == INVALID, bad and (bad.features, bad.in_pitch, bad.out_pitch)
    assert call(lib, z=z(136, 0, 0)) == call(lib, z=z(136, 0, 144)) == UNSUPPORTED
    for good in (z(16, 0, 0), z(1 << 20, 0, 0), z(128, 136, 144), z(128, 128, 128)):
        assert call(lib, z=good) == DEVICE
    # Without a layout: every row, and no config.
    alone = dict(no_layout=True, cfg=None)
    assert call(lib, **alone) == call(lib, **alone, rows=1) == call(lib, **alone, rows=1 << 33) == DEVICE
    assert call(lib, **alone, rows=-1) == INVALID
    assert call(lib, **alone, rows=0, a=None, q=None, qs=None) == OK


def test_gated_fields(lib):
    call = CALLS["gated"]
    g = epl.Gated
    for inner in (0, 4, 12, -8, WIDE):
        assert call(lib, g=g(inner, 1, 0)) == INVALID, inner
    for act in (-1, 4):
        assert call(lib, g=g(64, act, 0)) == INVALID, act
    dense = 64 * 128
    for stride in (dense - 16, dense + 8, -16, 1 << 62, (1 << 63) - 1):
        assert call(lib, g=g(64, 1, stride)) == INVALID, stride
    for good in (g(64, 0, dense), g(64, 3, dense + 16), g(8, 1, 0), g(1 << 20, 1, 1 << 40)):
        assert call(lib, g=good) == DEVICE
    assert call(lib, g=None) == INVALID
    assert call(lib, cfg=epl.config(2, 8, 2, epl.MAX_INT8_FEATURES, 4)) == DEVICE
    assert call(lib, cfg=epl.config(2, 8, 2, epl.MAX_INT8_FEATURES + 16, 4)) == UNSUPPORTED
    assert 128 * 128 * epl.MAX_INT8_FEATURES < 2 ** 31 <= 128 * 128 * (epl.MAX_INT8_FEATURES + 16)


def test_linear_fields(lib):
    call = CALLS["linear"]
    bad = [dict(K=4), dict(N=12), dict(K=WIDE), dict(N=WIDE), dict(ip=112), dict(ip=136), dict(op=56), dict(op=68),
           dict(rp=56), dict(rp=68), dict(op=-64), dict(ip=WIDE), dict(act=4), dict(act=-1), dict(stride=128 * 64 - 16),
           dict(stride=128 * 64 + 8), dict(stride=1 << 62), dict(stride=-128 * 64)]
    for kw in bad:
        assert call(lib, l=lin(**kw)) == INVALID, kw
    assert call(lib, l=None) == INVALID
    for kw in (dict(ip=144), dict(op=72), dict(rp=72), dict(stride=128 * 64 + 16), dict(N=8), dict(N=1 << 20),
               dict(K=epl.MAX_INT8_FEATURES), dict(payload=1), dict(payload=9)):
        assert call(lib, l=lin(**kw)) == DEVICE, kw
    for K in (136, epl.MAX_INT8_FEATURES + 16, 1 << 20):
        assert call(lib, l=lin(K=K, stride=1 << 30)) == UNSUPPORTED, K
    assert call(lib, out="res", l=lin(rp=72)) == INVALID  # in place needs one pitch
    assert call(lib, out="res", l=lin(rp=72, op=72)) == DEVICE
