"""A row of an int8 product comes out the same, bit for bit, whatever rows it is called with: its sums are exact, and what
follows them are the same fp32 operations in the kernel for a handful of rows and on every tile shape."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import Packed

pytestmark = pytest.mark.gpu

# One expert, so rows an expert: the last call of the handful's kernel, then the ends of those of 64, 128 and 256 rows a tile.
ROWS = (16, 17, 55, 56, 143, 144, 300)


def bits(t):
    return t.cpu().view(torch.int16)


def inputs(K, N, seed):
    g, dev = torch.Generator().manual_seed(seed), device()
    x = torch.randint(-127, 128, (ROWS[-1], K), generator=g, dtype=torch.int8)
    x[3] = 0  # sums of zero, with a scale below zero: the sign of what comes out
    xs = torch.rand(ROWS[-1], generator=g) * 0.02 + 0.001
    xs[::3] *= -1  # a weight in the scale may be
    w = torch.randint(-127, 128, (1, N, K), generator=g, dtype=torch.int8)
    ws = torch.rand(1, N, generator=g) * 0.02 + 0.001
    return g, dev, x.to(dev), xs.to(dev), w.to(dev), ws.to(dev)


def with_rows(T):
    return Packed(np.zeros((T, 1), np.int32), 1, 64, device())


@pytest.mark.parametrize("K,N", [(16, 8), (272, 520), (2064, 264)])
@pytest.mark.parametrize("activation", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("residual", [False, True])
def test_linear(K, N, activation, biased, residual):
    g, dev, x, xs, w, ws = inputs(K, N, K)
    bias = torch.randn(1, N, generator=g).bfloat16().to(dev) if biased else None
    res = torch.randn(ROWS[-1], N, generator=g).bfloat16().to(dev)
    out = []
    for T in ROWS:
        pk = with_rows(T)
        out.append(epl.experts_linear_int8(pk.cfg, x[:T], xs[:T], pk.L, w, ws, bias, res[:T] if residual else None, activation))
    torch.cuda.synchronize()
    for T, o in zip(ROWS, out):
        assert torch.equal(bits(o[:T]), bits(out[-1][:T])), "%d rows" % T


@pytest.mark.parametrize("K,N", [(16, 8), (272, 520), (2064, 264)])
@pytest.mark.parametrize("activation", ["none", "silu", "gelu", "relu"])
def test_gated(K, N, activation):
    g, dev, x, xs, w, ws = inputs(K, N, K + 1)
    up = torch.randint(-127, 128, w.shape, generator=g, dtype=torch.int8).to(dev)
    out = []
    for T in ROWS:
        pk = with_rows(T)
        cfg = epl.config(1, 1, 1, K, T)
        out.append(epl.experts_gated_int8(cfg, x[:T], xs[:T], pk.L, w, ws, up, ws, activation))
    torch.cuda.synchronize()
    for T, o in zip(ROWS, out):
        assert torch.equal(bits(o[:T]), bits(out[-1][:T])), "%d rows" % T
