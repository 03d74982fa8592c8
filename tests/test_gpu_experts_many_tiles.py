"""The products where a workgroup takes more than one tile (more than 512 tiles, a launch has at most 256 workgroups), on
every tile shape: the next tile's first steps are loaded before this one's results are stored, and what a step waits for
counts those stores, one, two or three for each group of columns. And the E4M3 linear product on each of its kernels.

Against 64 bits, worked out on the GPU expert by expert, within the bounds of products_util; NaN behind the last row and in
the gaps of the inputs, markers in the outputs; ragged row counts and odd features; reductions of three to twelve steps."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import (FEW, SLOPE, Packed, act, act_grad, dequantise_rows, dequantise_weights, quantise_rows,
                                 quantise_weights, rounded, routing_of_counts, sum_error, weights)

pytestmark = pytest.mark.gpu


def within(got, want, bound, what):
    """assert_within of products_util without the way to the host."""
    assert bool(torch.isfinite(got).all()), what + ": not finite"
    over = (got.double() - want).abs() - bound
    i = int(over.argmax())
    assert float(over.flatten()[i]) <= 0, "%s: element %d is %.9g, expected %.9g +- %.3g" % (
        what, i, got.flatten()[i], want.flatten()[i], bound.flatten()[i])


def layer(E, rows, H, seed, payload="bf16", pitch=0, padded=5):
    """E experts of about `rows` rows each (some a little more or less), one without rows, and padded tokens."""
    rng = np.random.default_rng(seed)
    counts = [int(c) for c in rows + rng.integers(-rows // 16, rows // 16 + 1, E)]
    if E > 4:
        counts[E // 2] = 0
    idx = np.concatenate([routing_of_counts(counts, E, 1, rng), np.full((padded, 1), -1, np.int32)])
    return Packed(idx, E, H, device(), payload=payload, row_pitch=pitch)


def tiles(pk, BM, columns, BN):
    return sum(-(-(b - a) // BM) for _, a, b in pk.experts()) * -(-columns // BN)


def check_gated(pk, x, wg, wu, name, h, pre):
    """x and the weights as 64-bit tensors, or functions of the expert that give them."""
    I = h.shape[1]
    for e, a, b in pk.experts():
        if a == b:
            continue
        xe, g_w, u_w = x[a:b].double(), wg(e), wu(e)
        K = xe.shape[1]
        g, u = xe @ g_w.T, xe @ u_w.T
        dg = sum_error(K + 2, xe.abs() @ g_w.abs().T) + FEW * g.abs()
        du = sum_error(K + 2, xe.abs() @ u_w.abs().T) + FEW * u.abs()
        v = act(name, g)
        err = SLOPE * dg * (u.abs() + du) + (v.abs() + FEW) * du + FEW * (v * u).abs()
        within(h[a:b], v * u, rounded(v * u, err), "h of expert %d" % e)
        within(pre[a:b, :I], g, rounded(g, dg), "gate projections of expert %d" % e)
        within(pre[a:b, I:], u, rounded(u, du), "up projections of expert %d" % e)
    pk.assert_untouched(h, "h")
    pk.assert_untouched(pre, "pre")


def check_linear(pk, x, w, bias, res, name, out, pre):
    for e, a, b in pk.experts():
        if a == b:
            continue
        xe, we, be, re = x[a:b].double(), w(e), bias[e].double(), res[a:b].double()
        K = xe.shape[1]
        v = xe @ we.T + be
        err = sum_error(K + 4, xe.abs() @ we.abs().T) + FEW * (v.abs() + be.abs())
        within(pre[a:b], v, rounded(v, err), "pre of expert %d" % e)
        y = act(name, v)
        err = SLOPE * err + FEW * y.abs()
        within(out[a:b], y + re, rounded(y + re, err + FEW * ((y + re).abs() + re.abs())), "out of expert %d" % e)
    pk.assert_untouched(out, "out")
    pk.assert_untouched(pre, "pre")


# experts, rows each, features out, tile rows: the 128-row tiles and the 256-row ones
BF16 = {"128": (8, 310, 128 * 26 + 8, 128), "256": (2, 2200, 128 * 29 + 8, 256)}


@pytest.mark.parametrize("K", [136, 264, 456])
@pytest.mark.parametrize("shape", BF16)
def test_gated(shape, K):
    E, rows, I, BM = BF16[shape]
    g = torch.Generator().manual_seed(K)
    pk = layer(E, rows, K, K, pitch=512)
    assert (pk.rows // E >= 1024) == (BM == 256) and tiles(pk, BM, I, 128) > 512
    x, wg, wu = pk.buffer(g, K, 512), weights(g, E, I, K, pk.dev), weights(g, E, I, K, pk.dev)
    name = {136: "silu", 264: "gelu", 456: "relu"}[K]
    h, pre = pk.out(I), pk.out(2 * I)
    epl.experts_gated(pk.cfg, x, pk.L, wg, wu, name, h=h, pre=pre)
    alone, _ = epl.experts_gated(pk.cfg, x, pk.L, wg, wu, name)  # a third of the stores
    torch.cuda.synchronize()
    assert torch.equal(alone[: pk.P], h[: pk.P])
    check_gated(pk, x, lambda e: wg[e].double(), lambda e: wu[e].double(), name, h, pre)


@pytest.mark.parametrize("name", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("shape,N", [("128", 256 * 24 + 72), ("256", 256 * 29 + 8)])
def test_linear(shape, N, name):
    E, rows, _, BM = BF16[shape]
    K = {"none": 200, "silu": 264, "gelu": 136, "relu": 520}[name]
    g = torch.Generator().manual_seed(N + K)
    pk = layer(E, rows, 64, N)
    assert (pk.rows // E >= 1024) == (BM == 256) and tiles(pk, BM, N, 256) > 512
    x, w = pk.buffer(g, K, K + 8), weights(g, E, N, K, pk.dev, N * K + 16)
    bias, res = torch.randn(E, N, generator=g).bfloat16().to(pk.dev), pk.buffer(g, N, N + 24)
    out, pre = pk.out(N, N + 64), pk.out(N)
    epl.experts_linear(pk.cfg, x, pk.L, w, bias, res, name, out=out, pre=pre)
    alone, _ = epl.experts_linear(pk.cfg, x, pk.L, w, bias, res, name)  # half of the stores
    torch.cuda.synchronize()
    assert torch.equal(alone[: pk.P], out[: pk.P])
    check_linear(pk, x, lambda e: w[e].double(), bias, res, name, out, pre)


def quantised(g, pk, K, pitch=0):
    """Rows as the fp8 dispatch writes them, NaN behind the last; blocks of very different scales and a row of zeros."""
    x = torch.randn(pk.rows, K, generator=g)
    x[:, :128] *= 50.0
    x[0] = 0.0
    q, s = quantise_rows(x)
    q[pk.P:], s[pk.P:] = 0x7F, float("nan")
    buf = torch.full((pk.rows, pitch or K), 0x7F, dtype=torch.uint8)
    buf[:, :K] = q
    return buf.to(pk.dev)[:, :K], s.to(pk.dev)


def quantised_weights(g, E, N, K, dev):
    q, s = quantise_weights(torch.randn(E, N, K, generator=g) * K ** -0.5)
    q, s = q.to(dev), s.to(dev)
    return q, s, lambda e: dequantise_weights(q[e:e + 1], s[e:e + 1])[0]


# experts, rows each, tile rows: fewer than 256 rows an expert take 64-row tiles, more 128-row ones
E4M3 = {"64": (16, 230, 64), "128": (8, 310, 128)}


@pytest.mark.parametrize("K", [128, 512, 640])
@pytest.mark.parametrize("shape", E4M3)
def test_gated_fp8(shape, K):
    E, rows, BM = E4M3[shape]
    I = 128 * (10 if BM == 64 else 26) + 40
    g = torch.Generator().manual_seed(K + BM)
    pk = layer(E, rows, K, K + 1, payload="fp8", pitch=640)
    assert (pk.rows // E < 256) == (BM == 64) and tiles(pk, BM, I, 128) > 512
    x, s = quantised(g, pk, K, 640)
    wg, sg, wide_g = quantised_weights(g, E, I, K, pk.dev)
    wu, su, wide_u = quantised_weights(g, E, I, K, pk.dev)
    h, pre = pk.out(I), pk.out(2 * I)
    epl.experts_gated(pk.cfg, x, pk.L, wg, wu, "silu", s, sg, su, h, pre)
    alone, _ = epl.experts_gated(pk.cfg, x, pk.L, wg, wu, "silu", s, sg, su)
    torch.cuda.synchronize()
    assert torch.equal(alone[: pk.P], h[: pk.P])
    check_gated(pk, dequantise_rows(x[: pk.P], s[: pk.P]), wide_g, wide_u, "silu", h, pre)


@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
@pytest.mark.parametrize("shape", ["few", "64", "128"])
def test_linear_fp8(shape, name):
    E, rows, BM = E4M3.get(shape, (8, 2, 16))
    K = {"none": 128, "gelu": 512, "silu": 896}[name]
    N = 256 * {"few": 1, "64": 9, "128": 26}[shape] + 40
    g = torch.Generator().manual_seed(K + E)
    pk = layer(E, rows, 64, K + 2, padded=2 if shape == "few" else 5)
    if shape == "few":
        assert pk.rows <= 16
    else:
        assert pk.rows > 16 and (pk.rows // E < 256) == (BM == 64) and tiles(pk, BM, N, 256) > 512
    x, s = quantised(g, pk, K, K + 16)
    w, sw, wide = quantised_weights(g, E, N, K, pk.dev)
    bias, res = torch.randn(E, N, generator=g).bfloat16().to(pk.dev), pk.buffer(g, N, N + 24)
    out, pre = pk.out(N, N + 8), pk.out(N)
    epl.experts_linear(pk.cfg, x, pk.L, w, bias, res, name, s, sw, out, pre)
    alone, _ = epl.experts_linear(pk.cfg, x, pk.L, w, bias, res, name, s, sw)
    torch.cuda.synchronize()
    assert torch.equal(alone[: pk.P], out[: pk.P])
    check_linear(pk, dequantise_rows(x[: pk.P], s[: pk.P]), wide, bias, res, name, out, pre)


@pytest.mark.parametrize("I", [136, 264])
def test_gated_backward(I):
    """Two parts of the reduction in the gradient of the rows, and tiles of both weights' gradients."""
    E, rows, BM = 8, 310, 128
    H = 256 * 24 + 8
    g = torch.Generator().manual_seed(I)
    pk = layer(E, rows, H, I, pitch=H - H % 64 + 64)
    x, wg, wu = pk.buffer(g, H, pk.cfg.pitch), weights(g, E, I, H, pk.dev), weights(g, E, I, H, pk.dev)
    assert tiles(pk, BM, H, 256) > 512 and E * 2 * -(-I // 128) * 25 > 512
    dh, pre = pk.buffer(g, I), pk.buffer(g, 2 * I)
    dx, dpre = pk.out(H, pk.cfg.pitch), pk.out(2 * I)
    _, dwg, dwu = epl.experts_gated_backward(pk.cfg, dh, pre, x, pk.L, wg, wu, dpre=dpre, drecv=dx)
    torch.cuda.synchronize()
    pk.assert_untouched(dx, "drecv")
    for e, a, b in pk.experts():
        if a == b:
            assert not dwg[e].any() and not dwu[e].any()
            continue
        xe, d, p = x[a:b].double(), dh[a:b].double(), pre[a:b].double()
        gg, u = p[:, :I], p[:, I:]
        dg, du = d * u * act_grad("silu", gg), d * act("silu", gg)
        eg, eu = rounded(dg, FEW * (d * u).abs() * SLOPE), rounded(du, FEW * (d * gg).abs())
        wge, wue = wg[e].double(), wu[e].double()
        want = dg @ wge + du @ wue
        err = eg @ wge.abs() + eu @ wue.abs() + sum_error(
            2 * I + 2, (dg.abs() + eg) @ wge.abs() + (du.abs() + eu) @ wue.abs())
        within(dx[a:b], want, rounded(want, err), "drecv of expert %d" % e)
        for got, dd, ee, what in ((dwg, dg, eg, "dw_gate"), (dwu, du, eu, "dw_up")):
            want = dd.T @ xe
            err = ee.T @ xe.abs() + sum_error(b - a + 2, (dd.abs() + ee).T @ xe.abs())
            within(got[e], want, rounded(want, err), "%s of expert %d" % (what, e))


def test_linear_backward():
    E, rows, K, N = 8, 310, 256 * 24 + 8, 264
    g = torch.Generator().manual_seed(31)
    pk = layer(E, rows, 64, 31)
    a_, w = pk.buffer(g, K, K + 8), weights(g, E, N, K, pk.dev)
    dy, pre = pk.buffer(g, N, N + 8), pk.buffer(g, N)
    assert tiles(pk, 128, K, 256) > 512 and E * -(-N // 128) * 25 > 512
    da = pk.out(K, K + 8)
    _, dw, db = epl.experts_linear_backward(pk.cfg, dy, a_, pk.L, w, pre, "silu", need_dbias=True, da=da)
    torch.cuda.synchronize()
    pk.assert_untouched(da, "da")
    for e, a, b in pk.experts():
        if a == b:
            assert not dw[e].any() and not db[e].any()
            continue
        x, we, d0 = a_[a:b].double(), w[e].double(), dy[a:b].double()
        d = d0 * act_grad("silu", pre[a:b].double())
        sums = FEW * d0.abs() * SLOPE
        er = rounded(d, sums)
        want = d @ we
        within(da[a:b], want, rounded(want, er @ we.abs() + sum_error(N + 2, (d.abs() + er) @ we.abs())), "da")
        want = d.T @ x
        within(dw[e], want, rounded(want, er.T @ x.abs() + sum_error(b - a + 2, (d.abs() + er).T @ x.abs())), "dw")
        want = d.sum(0)
        within(db[e], want, rounded(want, sums.sum(0) + sum_error(b - a + 2, d.abs().sum(0))), "dbias")


def test_pitches_past_32_bits_are_refused():
    """Rows 2^32 + 64 elements apart (one buffer of 8.6 GB): the C structs hold 32 bits, of which 64 would be left."""
    pk = Packed(np.zeros((2, 1), np.int32), 1, 64, device())
    pitch = 2 ** 32 + 64
    far = torch.empty(pitch + 64, dtype=torch.bfloat16, device=pk.dev).as_strided((2, 64), (pitch, 1))
    near = torch.zeros(2, 64, dtype=torch.bfloat16, device=pk.dev)
    w = torch.zeros(1, 64, 64, dtype=torch.bfloat16, device=pk.dev)
    for kw in (dict(a=far), dict(residual=far), dict(out=far)):
        with pytest.raises(epl.EplError, match="INVALID"):
            epl.experts_linear(pk.cfg, kw.pop("a", near), pk.L, w, **kw)
    # (Gradients of rows so far apart would be as large again.)
    for kw in (dict(dy=far), dict(a=far, da=far)):
        with pytest.raises(epl.EplError, match="INVALID"):
            epl.experts_linear_backward(pk.cfg, kw.pop("dy", near), kw.pop("a", near), pk.L, w, **kw)
