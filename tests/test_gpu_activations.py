"""The products' activations and their derivatives point by point, relative to the result: at every bf16 value, also far
out, where an activation is a small difference from zero. A product with one entry of one in each row of the weights
hands every kernel an exact argument.

Bounds, besides the rounding to bf16. GELU v Phi(v) = v erfc(x) / 2, x = -v / sqrt 2: x has a rounded constant and a
rounded product, 2 units of 2^-24, and erfc multiplies a relative error of x by at most 2 x^2 + 2 = v^2 + 2; the functions
and products add at most 16 units. The derivatives cross zero, GELU's is a published polynomial (evaluated at every bf16
value in 32 bits it is off by 4e-4 of the result at most) and SiLU's a sum with one rounding of its terms (1e-4): both are
given 2^-10, a quarter of the rounding to bf16. Below fp32's normal range nothing is asked."""
import math

import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import BF16_HALF_STEP, FEW, Packed

pytestmark = pytest.mark.gpu

FLOOR = 2.0 ** -126
ONE = 0x38  # 1.0 in E4M3


def points(limit):
    """Every bf16 value of magnitude 2^-20 to limit, both signs, and the zeros."""
    bits = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16)
    v = v[(v.float() >= 2.0 ** -20) & (v.float() <= limit)]
    return torch.cat([v, -v, torch.tensor([0.0, -0.0], dtype=torch.bfloat16)])


def exact(name, v):
    """act(v), act'(v) and what an fp32 act(v) may be off by, in 64 bits."""
    v = v.double()
    if name == "silu":
        s, c = torch.sigmoid(v), torch.sigmoid(-v)
        return v * s, s * (1 + v * c), FEW * (v * s).abs()
    if name == "gelu":
        phi, cdf = torch.exp(-v * v / 2) / math.sqrt(2 * math.pi), torch.special.erfc(-v / math.sqrt(2)) / 2
        return v * cdf, cdf + v * phi, (FEW + 2.0 ** -23 * (v * v + 2)) * (v * cdf).abs()
    if name == "relu":
        return v.clamp_min(0), (v > 0).double(), torch.zeros_like(v)
    return v, torch.ones_like(v), torch.zeros_like(v)


def assert_close(got, want, err, what, at):
    got = got.cpu().double()
    over = (got - want).abs() - (err + BF16_HALF_STEP * (want.abs() + err) + FLOOR)
    i = int(over.argmax())
    assert float(over[i]) <= 0, "%s at %.9g: %.9g, expected %.9g" % (what, at[i], got[i], want[i])


def rows_of(v, E):
    """A layout of len(v) rows, one choice each, dealt to E experts; row r's value is its r-th."""
    T = v.numel()
    idx = (np.arange(T) * E // T).astype(np.int32)[:, None]
    return Packed(idx, E, 128, device())


def one_hot(E, N, K, at, dev):
    w = torch.zeros(E, N, K, dtype=torch.bfloat16, device=dev)
    w[:, :, at] = 1.0
    return w


# 256 x 256 tiles, 128 x 256 tiles, the form for few rows; fp8: 128- and 64-row tiles, few rows.
KERNELS = [("bf16", 1), ("bf16", 8), ("bf16", 16), ("fp8", 8), ("fp8", 64), ("fp8", 16)]
LIMIT = {"silu": 100.0, "gelu": 14.0, "relu": 1e30, "none": 1e30}


@pytest.mark.parametrize("payload,E", KERNELS, ids=lambda p: str(p))
@pytest.mark.parametrize("name", ["silu", "gelu", "relu", "none"])
def test_forward(name, payload, E):
    v = points(LIMIT[name]) if name in ("silu", "gelu") else points(100.0)
    if E == 16:
        v = torch.linspace(-LIMIT[name] * 0.9, LIMIT[name] * 0.1, 16).bfloat16() if name in ("silu", "gelu") else v[::500][:16]
    pk = rows_of(v, E)
    d, T, N = pk.dev, v.numel(), 8
    cap, per = T, T // E
    assert (cap <= 16) == (E == 16) and (E != 1 or per >= 1024) and (E != 8 or 256 <= per < 1024) and (E != 64 or per < 256)
    want, _, err = exact(name, v)
    if payload == "bf16":
        x = torch.zeros(T, 128, dtype=torch.bfloat16)
        x[:, 0], x[:, 1] = v, 1.0
        x = x.to(d)
        out, pre = epl.experts_linear(pk.cfg, x, pk.L, one_hot(E, N, 128, 0, d), activation=name, keep_pre=True)
        h, _ = epl.experts_gated(pk.cfg, x, pk.L, one_hot(E, N, 128, 0, d), one_hot(E, N, 128, 1, d), activation=name)
    else:
        x = torch.zeros(T, 128, dtype=torch.uint8)
        x[:, 0] = ONE
        w = torch.zeros(E, N, 128, dtype=torch.uint8)
        w[:, :, 0] = ONE
        s, ws = v.float()[:, None].to(d), torch.ones(E, N, device=d)
        x, w = x.to(d), w.to(d)
        out, pre = epl.experts_linear(pk.cfg, x, pk.L, w, activation=name, a_scale=s, w_scale=ws, keep_pre=True)
        # The up projection of the same rows is v itself: divided out below.
        cfg = epl.config(1, E, 1, 128, T, "fp8")
        h, _ = epl.experts_gated(cfg, x, pk.L, w, w, name, s, ws, ws)
    torch.cuda.synchronize()
    assert torch.equal(pre.cpu()[:, 0], v)
    assert bool((out == out[:, :1]).all()) and bool((h == h[:, :1]).all())
    assert_close(out[:, 0], want, err, name, v)
    if payload == "bf16":
        assert_close(h[:, 0], want, err + FEW * want.abs(), "gated " + name, v)
    else:
        up = v.double()
        assert_close(h[:, 0], want * up, (err + FEW * want.abs()) * up.abs() + FLOOR * up.abs(), "gated " + name, v)


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_gradient(name):
    v = points(LIMIT[name]) if name != "relu" else points(100.0)
    pk = rows_of(v, 8)
    d, T, N = pk.dev, v.numel(), 8
    act, grad, err = exact(name, v)
    slack = 2.0 ** -10 * grad.abs()
    x = torch.zeros(T, 8, dtype=torch.bfloat16, device=d)
    w = torch.zeros(8, N, 8, dtype=torch.bfloat16, device=d)
    pre = v[:, None].expand(T, N).contiguous().to(d)
    dy = torch.ones(T, N, dtype=torch.bfloat16, device=d)
    for need_dbias in (False, True):  # two kernels
        dpre = torch.empty(T, N, dtype=torch.bfloat16, device=d)
        epl.experts_linear_backward(pk.cfg, dy, x, pk.L, w, pre, name, need_dbias=need_dbias, dpre=dpre)
        torch.cuda.synchronize()
        assert bool((dpre == dpre[:, :1]).all())
        assert_close(dpre[:, 0], grad, slack, name + "'", v)
    cfg = epl.config(1, 8, 1, 8, T)
    both = torch.cat([pre, torch.ones_like(pre)], 1)  # u = 1
    dpre = torch.empty(T, 2 * N, dtype=torch.bfloat16, device=d)
    epl.experts_gated_backward(cfg, dy, both, x, pk.L, w, w, name, dpre=dpre)
    torch.cuda.synchronize()
    assert_close(dpre[:, 0], grad, slack, "gate " + name + "'", v)
    assert_close(dpre[:, N], act, err + FEW * act.abs(), "up " + name, v)
