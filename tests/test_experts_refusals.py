"""Refusals of the products, the router and combine's gradient on the host, from a call that is right in everything but
one argument: the unchanged call passes every check (its status is then that of a launch where there is no device), so a
refusal is the argument's. The pointers are fake addresses: on a machine with a GPU the unchanged calls would launch, so
nothing runs there."""
import ctypes
import os

import pytest
import torch

from paper_2607_06202_amd import epl

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are fake, and a GPU would follow them")

OK, INVALID, ALIGN, CAPACITY, UNSUPPORTED, DEVICE = 0, 1, 2, 3, 5, 6
P = 0x10000
CFG = epl.config(2, 8, 2, 128, 4)  # T = 8, T*k = 16
FP8 = epl.config(2, 8, 2, 128, 4, "fp8")
EMPTY = epl.config(2, 8, 2, 128, 0)
one = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(epl.LIB_PATH):
        from paper_2607_06202_amd import _build
        _build.build()
    return epl.lib()


def layout(at=64):
    """Layout buffers at addresses of their own; expert_off and pair_row among the calls' inputs."""
    return {n: (at + i) * P for i, (n, _) in enumerate(epl.LayoutBuffers._fields_)}


def lin(K=128, N=64, ip=0, op=0, rp=0, act=1, payload=0, stride=0):
    return epl.Linear(K, N, ip, op, rp, act, payload, stride)


class Call:
    """An entry point with every buffer at an address of its own. call(name=value) changes that argument; a value that
    names another buffer stands for its address."""

    def __init__(self, name, buffers, config, inputs, outputs, may=()):
        self.name, self.config = name, config
        self.inputs, self.outputs = inputs.split(), outputs.split()
        self.may = {frozenset(m) for m in may}  # pairs that may be one buffer
        self.at = dict({n: (i + 1) * P for i, n in enumerate(buffers.split())}, **layout())

    def pairs(self):
        """Each output with each input and each other output, without the documented ones."""
        for i, o in enumerate(self.outputs):
            for other in self.inputs + self.outputs[:i]:
                if frozenset((o, other)) not in self.may:
                    yield o, other

    def __call__(self, lib, **kw):
        v = dict(self.config, rows=16, **self.at)
        v.update({n: v[x] if isinstance(x, str) else x for n, x in kw.items()})
        L = epl.LayoutBuffers(*[v[n] for n, _ in epl.LayoutBuffers._fields_])
        return ARGS[self.name](lib, v, L)


ARGS = {
    "gated": lambda lib, v, L: lib.epl_experts_gated(
        one(v["cfg"]), one(epl.Gated(v["inner"], v["act"], v["stride"])), v["recv"], v["rs"], v["rows"], one(L), v["wg"],
        v["wu"], v["gs"], v["us"], v["h"], v["pre"], None),
    "gated_backward": lambda lib, v, L: lib.epl_experts_gated_backward(
        one(v["cfg"]), one(epl.Gated(v["inner"], v["act"], v["stride"])), v["dh"], v["pre"], v["recv"], v["rows"], one(L),
        v["wg"], v["wu"], v["dpre"], v["drecv"], v["dwg"], v["dwu"], None),
    "linear": lambda lib, v, L: lib.epl_experts_linear(
        one(v["cfg"]), one(v["l"]), v["a"], v["asc"], v["rows"], one(L), v["w"], v["wsc"], v["bias"], v["res"], v["out"],
        v["pre"], None),
    "linear_backward": lambda lib, v, L: lib.epl_experts_linear_backward(
        one(v["cfg"]), one(v["l"]), v["dy"], v["pre"], v["a"], v["rows"], one(L), v["w"], v["dpre"], v["da"], v["dw"],
        v["db"], None),
    "route": lambda lib, v, L: lib.epl_route(one(v["cfg"]), one(v["o"]), v["logits"], v["bias"], v["idx"], v["w"], None),
    "route_backward": lambda lib, v, L: lib.epl_route_backward(
        one(v["cfg"]), one(v["o"]), v["logits"], v["idx"], v["dw"], v["dl"], None),
    "combine_backward": lambda lib, v, L: lib.epl_combine_backward(
        one(v["cfg"]), v["dout"], v["y"], v["w"], one(L), v["dy"], v["rows"], v["dw"], None),
}

GATED = dict(cfg=CFG, inner=64, act=1, stride=0)
CALLS = {
    "gated": Call("gated", "recv rs wg wu gs us h pre", GATED, "recv wg wu expert_off", "h pre"),
    "gated_fp8": Call("gated", "recv rs wg wu gs us h pre", dict(GATED, cfg=FP8), "recv rs wg wu gs us expert_off",
                      "h pre"),
    "gated_backward": Call("gated_backward", "dh pre recv wg wu dpre drecv dwg dwu", GATED,
                           "dh pre recv wg wu expert_off", "dpre drecv dwg dwu", [("dpre", "pre")]),
    "linear": Call("linear", "a asc w wsc bias res out pre", dict(cfg=CFG, l=lin()), "a w bias res expert_off",
                   "out pre", [("out", "res")]),
    "linear_fp8": Call("linear", "a asc w wsc bias res out pre", dict(cfg=CFG, l=lin(payload=1)),
                       "a asc w wsc bias res expert_off", "out pre", [("out", "res")]),
    "linear_backward": Call("linear_backward", "dy pre a w dpre da dw db", dict(cfg=CFG, l=lin()),
                            "dy pre a w expert_off", "dpre da dw db", [("dpre", "pre")]),
    # Without an activation pre and dpre are ignored.
    "linear_backward_none": Call("linear_backward", "dy pre a w dpre da dw db", dict(cfg=CFG, l=lin(act=0)),
                                 "dy a w expert_off", "da dw db"),
    "route": Call("route", "logits bias idx w", dict(cfg=CFG, o=epl.RouteOpts(0, 0, 1, 1.0)), "logits bias", "idx w"),
    "route_backward": Call("route_backward", "logits idx dw dl", dict(cfg=CFG, o=epl.RouteOpts(0, 0, 1, 1.0)),
                           "logits idx dw", "dl"),
    "combine_backward": Call("combine_backward", "dout y w dy dw", dict(cfg=CFG), "dout y w pair_row", "dy dw",
                             [("dy", "y")]),
}


@pytest.mark.parametrize("name", CALLS)
def test_an_output_at_the_address_of_another_buffer(lib, name):
    """Every output with every input and every other output: other workgroups, or a later launch of the same call, would
    read what was overwritten, or one result replace another."""
    call = CALLS[name]
    assert call(lib) == DEVICE
    for o, other in call.pairs():
        assert call(lib, **{o: other}) == INVALID, (o, other)
    for m in call.may:
        a, b = sorted(m)
        assert call(lib, **{a: b}) == DEVICE, (a, b)


def test_without_tokens_the_weights_gradients_are_still_written(lib):
    for name, o, other in (("gated_backward", "dwg", "dwu"), ("gated_backward", "dwu", "expert_off"),
                           ("linear_backward", "dw", "db"), ("linear_backward", "db", "expert_off")):
        assert CALLS[name](lib, cfg=EMPTY) == DEVICE
        assert CALLS[name](lib, cfg=EMPTY, **{o: other}) == INVALID, (name, o, other)
    assert CALLS["gated"](lib, cfg=EMPTY, h="recv") == OK  # nothing is read or written


WIDE = (1 << 20) + 8  # more features than EPL_MAX_HIDDEN


@pytest.mark.parametrize("name", CALLS)
def test_missing_and_misaligned_buffers(lib, name):
    """A buffer that the call uses is refused where it is null (unless optional) or misaligned; one that it ignores is
    not looked at."""
    call = CALLS[name]
    word = {"rs", "gs", "us", "asc", "wsc", "logits", "bias", "idx", "w", "dw", "dl", "expert_off", "pair_row"} \
        if "route" in name or name == "combine_backward" else {"rs", "gs", "us", "asc", "wsc", "expert_off"}
    if name == "combine_backward":
        word = {"w", "dw", "pair_row"}
    optional = {"gated": {"pre"}, "gated_fp8": {"pre"}, "linear": {"bias", "res", "pre"},
                "linear_fp8": {"bias", "res", "pre"}, "linear_backward": {"db"}, "linear_backward_none": {"db"},
                "route": {"bias"}}.get(name, set())
    used = call.inputs + call.outputs
    for n in used:
        assert call(lib, **{n: None}) == (DEVICE if n in optional else INVALID), n
        assert call(lib, **{n: call.at[n] + (2 if n in word else 8)}) == ALIGN, n
    for n in call.at:
        if n not in used:
            assert call(lib, **{n: None}) == call(lib, **{n: call.at[n] + 1}) == DEVICE, n


@pytest.mark.parametrize("name", CALLS)
def test_bad_configs_and_row_counts(lib, name):
    call = CALLS[name]
    for bad in (epl.config(3, 8, 2, 128, 4), epl.config(2, 8, 0, 128, 4), epl.config(2, 8, 2, 124, 4),
                epl.config(2, 8, 2, 128, -1)):
        assert call(lib, cfg=bad) == INVALID
    if "route" in name:
        return
    for rows in (15, 0, -1):
        assert call(lib, rows=rows) == CAPACITY
    assert call(lib, rows=17) == DEVICE


@pytest.mark.parametrize("name", ["gated", "gated_fp8", "gated_backward"])
def test_gated_fields(lib, name):
    call = CALLS[name]
    piece = 16 if "fp8" in name else 8  # elements of 16 bytes
    for inner in (0, 4, 12, -8, WIDE):
        assert call(lib, inner=inner) == INVALID, inner
    for act in (-1, 4):
        assert call(lib, act=act) == INVALID, act
    for act in range(4):
        assert call(lib, act=act) == DEVICE, act
    dense = 64 * 128
    for stride in (dense - piece, dense + piece // 2, -piece, 1 << 62, (1 << 63) - 1):
        assert call(lib, stride=stride) == INVALID, stride
    for stride in (0, dense, dense + piece, 1 << 40):
        assert call(lib, stride=stride) == DEVICE, stride
    assert call(lib, inner=8) == call(lib, inner=1 << 20) == DEVICE


def test_payloads(lib):
    assert CALLS["gated"](lib, cfg=epl.config(2, 8, 2, 136, 4, "fp8")) == UNSUPPORTED
    assert CALLS["gated_backward"](lib, cfg=FP8) == UNSUPPORTED
    assert CALLS["linear"](lib, l=lin(payload=2)) == UNSUPPORTED
    assert CALLS["linear"](lib, l=lin(K=64, payload=1)) == UNSUPPORTED
    assert CALLS["linear_backward"](lib, l=lin(payload=1)) == UNSUPPORTED
    assert CALLS["combine_backward"](lib, cfg=FP8) == DEVICE  # its rows are bf16 whatever the payload


@pytest.mark.parametrize("name", ["linear", "linear_fp8", "linear_backward", "linear_backward_none"])
def test_linear_fields(lib, name):
    call = CALLS[name]
    fp8 = "fp8" in name
    own = dict(payload=int(fp8), act=0 if "none" in name else 1)
    bad = [dict(K=4), dict(N=12), dict(K=WIDE, ip=0), dict(N=WIDE), dict(ip=120), dict(ip=132), dict(op=56),
           dict(op=68), dict(rp=56), dict(rp=68), dict(op=-64), dict(ip=WIDE), dict(act=4), dict(act=-1),
           dict(stride=128 * 64 - 16), dict(stride=128 * 64 + 4), dict(stride=1 << 62), dict(stride=-128 * 64)]
    if fp8:
        bad += [dict(ip=136), dict(stride=128 * 64 + 8)]  # E4M3 in 16-byte pieces
    for kw in bad:
        assert call(lib, l=lin(**{**own, **kw})) == INVALID, kw
    good = [dict(), dict(ip=128), dict(ip=144), dict(op=72), dict(rp=72), dict(stride=128 * 64), dict(stride=128 * 64 + 16),
            dict(N=8), dict(N=1 << 20), dict(K=1 << 20)]
    for kw in good:
        assert call(lib, l=lin(**{**own, **kw})) == DEVICE, kw
    if not name.startswith("linear_backward"):
        assert call(lib, out="res", l=lin(**own, rp=72)) == INVALID  # in place needs one pitch
        assert call(lib, out="res", l=lin(**own, rp=72, op=72)) == DEVICE


def test_route_fields(lib):
    nan, inf = float("nan"), float("inf")
    for name in ("route", "route_backward"):
        call = CALLS[name]
        for o in ((2, 0, 1, 1.0), (-1, 0, 1, 1.0), (0, 2, 1, 1.0), (0, -1, 1, 1.0), (0, 0, 2, 1.0), (0, 0, 1, nan),
                  (0, 0, 1, inf), (0, 0, 0, -inf)):
            assert call(lib, o=epl.RouteOpts(*o)) == INVALID, (name, o)
        for o in ((0, 0, 0, 1.0), (1, 1, 1, -2.5), (1, 0, 1, 0.0)):
            assert call(lib, o=epl.RouteOpts(*o)) == DEVICE, (name, o)
        assert call(lib, o=epl.RouteOpts(1, 0, 1, 1.0), logits=call.at["logits"] + 2) == DEVICE  # bf16
        assert call(lib, o=epl.RouteOpts(1, 0, 1, 1.0), logits=call.at["logits"] + 1) == ALIGN


def test_missing_structs(lib):
    L = epl.LayoutBuffers(*layout().values())
    g, l = epl.Gated(64, 1, 0), lin()
    p = [i * P for i in range(1, 12)]
    assert lib.epl_experts_gated(one(CFG), None, p[0], None, 16, one(L), p[1], p[2], None, None, p[3], None, None) == INVALID
    assert lib.epl_experts_gated(one(CFG), one(g), p[0], None, 16, None, p[1], p[2], None, None, p[3], None, None) == INVALID
    assert lib.epl_experts_gated(None, one(g), p[0], None, 16, one(L), p[1], p[2], None, None, p[3], None, None) == INVALID
    assert lib.epl_experts_linear(one(CFG), None, p[0], None, 16, one(L), p[1], None, None, None, p[2], None, None) == INVALID
    assert lib.epl_experts_linear(one(CFG), one(l), p[0], None, 16, None, p[1], None, None, None, p[2], None, None) == INVALID
    assert lib.epl_combine_backward(one(CFG), p[0], p[1], p[2], None, p[3], 16, p[4], None) == INVALID
    assert lib.epl_route(one(CFG), None, p[0], None, p[1], p[2], None) == INVALID


def test_without_tokens_nothing_but_weights_is_needed(lib):
    for name, needed in (("gated", ()), ("gated_fp8", ()), ("linear", ()), ("linear_fp8", ()), ("route", ()),
                         ("route_backward", ()), ("combine_backward", ()), ("gated_backward", ("dwg", "dwu")),
                         ("linear_backward", ("dw",))):
        call = CALLS[name]
        cfg = epl.config(2, 8, 2, 128, 0, "fp8" if name == "gated_fp8" else "bf16")
        none = {n: None for n in call.inputs + call.outputs if n not in needed and n not in ("expert_off", "pair_row")}
        assert call(lib, cfg=cfg, rows=0, **none) == (DEVICE if needed else OK), name
        for n in needed:
            assert call(lib, cfg=cfg, rows=0, **none, **{n: None}) == INVALID, (name, n)


def test_counts_past_32_bits_do_not_lose_their_upper_half():
    assert epl.Linear(64, 64, 2 ** 32 + 64, 0, 0, 0, 0, 0).in_pitch == 64  # what ctypes makes of it
    assert epl._int32(2 ** 31 - 1, "pitch") == 2 ** 31 - 1
    for v in (2 ** 31, 2 ** 32 + 64):
        with pytest.raises(epl.EplError, match="INVALID"):
            epl._int32(v, "pitch")
