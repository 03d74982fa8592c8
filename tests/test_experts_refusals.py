"""Refusals of the products, the router and combine's gradient on the host, from a call that is right in everything but one argument: the unchanged call
passes every check (its status is then that of a launch where there is no device), so a refusal is the argument's.
The pointers are fake addresses: on a machine with a GPU the unchanged calls would launch, so nothing runs there."""
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
