"""Inputs, 64-bit references and error bounds of the experts' products, the router and combine's gradient.

Bounds. A result that is summed in fp32 over n products and rounded to bf16 once is off by at most
    n * 2^-23 * sum |terms|   (each addition by at most one unit of 2^-23, whatever its rounding)
  + 2^-8 * |result|           (the rounding: half a bf16 step, finfo(bfloat16).eps / 2)
and what an activation does to the error of its argument follows from |act'| <= 1.13 (GELU's largest slope;
SiLU's is 1.1). Elementary functions and the few products around them add at most 16 units of 2^-24.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2607_06202_amd import epl

BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2
FEW = 16 * 2.0 ** -24
SLOPE = 1.13
TINY = 1e-37  # results below fp32's normal range


def act(name, v):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v / math.sqrt(2)))
    return v.clamp_min(0) if name == "relu" else v


def act_grad(name, v):
    if name == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(v / math.sqrt(2))) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    return (v > 0).double() if name == "relu" else torch.ones_like(v)


def sum_error(n: int, terms: torch.Tensor) -> torch.Tensor:
    return n * 2.0 ** -23 * terms


def rounded(value: torch.Tensor, error: torch.Tensor) -> torch.Tensor:
    """Bound of a bf16 result whose fp32 value is within error of value."""
    return error + BF16_HALF_STEP * (value.abs() + error) + TINY


def assert_within(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor, what: str) -> None:
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what + ": not finite"
    over = (got - want).abs() - bound
    if got.numel() and float(over.max()) > 0:
        i = int(over.argmax())
        raise AssertionError("%s: element %d is %.9g, expected %.9g +- %.3g" % (
            what, i, got.flatten()[i], want.flatten()[i], bound.flatten()[i]))


def routing_of_counts(counts, E: int, k: int, rng) -> np.ndarray:
    """[T, k] expert ids in which expert e occurs counts[e] times (places left over are -1), shuffled."""
    ids = np.repeat(np.arange(E), counts)
    T = max(1, -(-len(ids) // k))
    flat = np.full(T * k, -1, np.int32)
    flat[: len(ids)] = ids
    rng.shuffle(flat)
    return flat.reshape(T, k)


class Packed:
    """A layout on the GPU and what the tests know of it on the host."""

    def __init__(self, idx: np.ndarray, E: int, H: int, dev, R: int = 1, payload="bf16", row_pitch=0):
        T, k = idx.shape
        self.cfg = epl.config(R, E, k, H, T // R, payload, row_pitch)
        self.L = epl.layout(self.cfg, torch.from_numpy(np.ascontiguousarray(idx, np.int32)).to(dev))
        self.off = self.L.expert_off.cpu().tolist()
        self.P = self.off[-1]
        self.rows = T * k
        self.dev = dev

    def experts(self):
        return [(e, self.off[e], self.off[e + 1]) for e in range(self.cfg.num_experts)]

    def buffer(self, g, width, pitch=0, std=1.0, scatter_nan=True):
        """[rows, width] bf16 with rows pitch apart: values in rows 0..P-1, NaN behind them and in the gaps."""
        b = torch.full((self.rows, pitch or width), float("nan"), dtype=torch.bfloat16)
        b[: self.P, :width] = (torch.randn(self.P, width, generator=g) * std).bfloat16()
        return b.to(self.dev)[:, :width]

    def out(self, width, pitch=0):
        """An output buffer of a recognisable value, to see what is left untouched."""
        return torch.full((self.rows, pitch or width), 77.0, dtype=torch.bfloat16, device=self.dev)[:, :width]

    def assert_untouched(self, t: torch.Tensor, what: str) -> None:
        assert bool((t[self.P:] == 77.0).all()), what + ": rows behind the last were written"
        if t.stride(0) > t.shape[1]:
            whole = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))
            assert bool((whole[:, t.shape[1]:] == 77.0).all()), what + ": the gaps between rows were written"


def weights(g, E, N, K, dev, stride=0, std=None):
    """[E, N, K] bf16, the experts' matrices stride elements apart (NaN between them)."""
    w = (torch.randn(E, N, K, generator=g) * (std or K ** -0.5)).bfloat16()
    if not stride:
        return w.to(dev)
    b = torch.full((E, stride), float("nan"), dtype=torch.bfloat16)
    b[:, : N * K] = w.view(E, -1)
    return b.to(dev)[:, : N * K].view(E, N, K) if E == 1 else b.to(dev).as_strided((E, N, K), (stride, K, 1))


def quantise_rows(x: torch.Tensor):
    """E4M3 bytes and a scale per 128 elements."""
    b = x.float().view(x.shape[0], -1, 128)
    s = b.abs().amax(2) / 448
    q = (b / torch.where(s == 0, 1.0, s)[:, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).view(x.shape), s


def dequantise_rows(q, s):
    return q.contiguous().view(torch.float8_e4m3fn).double() * s.double().repeat_interleave(128, 1)


def quantise_weights(w: torch.Tensor):
    s = w.float().abs().amax(2) / 448
    return (w.float() / s[:, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s


def dequantise_weights(q, s):
    return q.view(torch.float8_e4m3fn).double() * s.double()[:, :, None]
