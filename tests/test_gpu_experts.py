"""The experts' products (epl_experts_gated, epl_experts_linear and their gradients) against 64-bit references, at
the sizes where a tile, a step of the reduction or a segment ends: experts without rows, with one row, with more
than a tile; rows behind the last one that hold NaN and must stay untouched; pitches, gaps between the experts'
matrices, features that are no multiple of a tile; every activation; the fp8 payload."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import (BF16_HALF_STEP, FEW, SLOPE, Packed, act, act_grad, assert_within, dequantise_rows,
                                 dequantise_weights, quantise_rows, quantise_weights, rounded, routing_of_counts,
                                 sum_error, weights)

pytestmark = pytest.mark.gpu

# Rows of each expert. The tile edges at 16, 32, 128 and 256 rows, empty and single-row experts.
COUNTS = {
    "one_token": [0, 0, 1, 0, 1, 0, 0, 1],
    "few": [3, 0, 1, 2, 0, 5, 16, 17],
    "edges": [127, 128, 129, 0, 1, 64, 255, 31],
    "one_expert": [0, 0, 0, 700, 0, 0, 0, 0],
    "none": [0, 0, 0, 0, 0, 0, 0, 0],
    "large": [513, 256, 300, 1, 0, 257, 640, 90],
}


def packed(counts, H, k=2, seed=0, **kw):
    rng = np.random.default_rng(seed)
    idx = routing_of_counts(COUNTS[counts], 8, k, rng)
    idx = np.concatenate([idx, np.full((3, k), -1, np.int32)])  # padded tokens
    return Packed(idx, 8, H, device(), **kw)


def gated_reference(pk, x, wg, wu, name):
    """h, pre and their bounds, in 64 bits, rows 0..P-1."""
    K = x.shape[1]
    I = wg.shape[1]
    h = torch.zeros(pk.P, I, dtype=torch.float64)
    hb = torch.zeros_like(h)
    pre = torch.zeros(pk.P, 2 * I, dtype=torch.float64)
    pb = torch.zeros_like(pre)
    for e, a, b in pk.experts():
        if a == b:
            continue
        xe = x[a:b]
        g, u = xe @ wg[e].T, xe @ wu[e].T
        dg = sum_error(K + 2, xe.abs() @ wg[e].abs().T) + FEW * g.abs()
        du = sum_error(K + 2, xe.abs() @ wu[e].abs().T) + FEW * u.abs()
        v = act(name, g)
        h[a:b] = v * u
        err = SLOPE * dg * (u.abs() + du) + (v.abs() + FEW) * du + FEW * (v * u).abs()
        hb[a:b] = rounded(v * u, err)
        pre[a:b] = torch.cat([g, u], 1)
        pb[a:b] = torch.cat([rounded(g, dg), rounded(u, du)], 1)
    return h, hb, pre, pb


CASES = [  # counts, H, I, pitch, activation, gap between matrices, halves of one tensor
    ("few", 8, 8, 0, "silu", 0, False),
    ("few", 200, 72, 256, "gelu", 0, True),
    ("one_token", 512, 264, 0, "silu", 0, False),
    ("edges", 136, 136, 192, "silu", 64, False),
    ("edges", 64, 128, 0, "relu", 0, True),
    ("one_expert", 328, 104, 0, "none", 0, False),
    ("none", 64, 64, 0, "silu", 0, False),
    ("large", 192, 296, 256, "silu", 0, True),
    ("large", 1032, 40, 0, "gelu", 8, False),
]


def gated_inputs(counts, H, I, pitch, gap, halves, seed):
    g = torch.Generator().manual_seed(seed)
    pk = packed(counts, H, row_pitch=pitch)
    x = pk.buffer(g, H, pitch)
    if halves:
        both = weights(g, 8, 2 * I, H, pk.dev)
        wg, wu = both[:, :I], both[:, I:]
    else:
        stride = I * H + gap if gap else 0
        wg, wu = weights(g, 8, I, H, pk.dev, stride), weights(g, 8, I, H, pk.dev, stride)
    return pk, x, wg, wu, g


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_gated_forward(case):
    counts, H, I, pitch, name, gap, halves = case
    pk, x, wg, wu, _ = gated_inputs(counts, H, I, pitch, gap, halves, 1)
    h, pre = pk.out(I), pk.out(2 * I)
    epl.experts_gated(pk.cfg, x, pk.L, wg, wu, name, h=h, pre=pre)
    alone, none = epl.experts_gated(pk.cfg, x, pk.L, wg, wu, name)
    torch.cuda.synchronize()
    assert none is None and torch.equal(alone[: pk.P], h[: pk.P])
    want, bound, wpre, pbound = gated_reference(pk, x[: pk.P].cpu().double(), wg.cpu().double(), wu.cpu().double(), name)
    assert_within(h[: pk.P], want, bound, "h")
    assert_within(pre[: pk.P], wpre, pbound, "pre")
    pk.assert_untouched(h, "h")
    pk.assert_untouched(pre, "pre")


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_gated_backward(case):
    counts, H, I, pitch, name, gap, halves = case
    pk, x, wg, wu, g = gated_inputs(counts, H, I, pitch, gap, halves, 2)
    pre, dh = pk.buffer(g, 2 * I), pk.buffer(g, I)
    dx = pk.out(H, pitch)
    dpre = pk.out(2 * I)
    _, dwg, dwu = epl.experts_gated_backward(pk.cfg, dh, pre, x, pk.L, wg, wu, name, dpre=dpre, drecv=dx)
    torch.cuda.synchronize()
    kept = pre.clone()
    dx2, dwg2, dwu2 = epl.experts_gated_backward(pk.cfg, dh, kept, x, pk.L, wg, wu, name, dpre=kept)  # in place
    torch.cuda.synchronize()
    assert torch.equal(dx2[: pk.P], dx[: pk.P]) and torch.equal(dwg, dwg2) and torch.equal(dwu, dwu2)
    pk.assert_untouched(dx, "drecv")
    pk.assert_untouched(dpre, "dpre")
    xd, wgd, wud = x.cpu().double(), wg.cpu().double(), wu.cpu().double()
    dhd, pd = dh.cpu().double(), pre.cpu().double()
    for e, a, b in pk.experts():
        if a == b:
            assert not dwg[e].any() and not dwu[e].any()
            continue
        gg, u, d = pd[a:b, :I], pd[a:b, I:], dhd[a:b]
        dg, du = d * u * act_grad(name, gg), d * act(name, gg)
        # dpre: its factors' roundings and act's and act''s own (relative to values below SLOPE and |g|), then bf16
        eg = rounded(dg, FEW * (d * u).abs() * SLOPE)
        eu = rounded(du, FEW * (d * gg).abs())
        assert_within(dpre[a:b, :I], dg, eg, "dpre gate")
        assert_within(dpre[a:b, I:], du, eu, "dpre up")
        want = dg @ wgd[e] + du @ wud[e]
        terms = (dg.abs() + eg) @ wgd[e].abs() + (du.abs() + eu) @ wud[e].abs()
        err = eg @ wgd[e].abs() + eu @ wud[e].abs() + sum_error(2 * I + 2, terms)
        assert_within(dx[a:b], want, rounded(want, err), "drecv")
        for got, dd, ee, what in ((dwg, dg, eg, "dw_gate"), (dwu, du, eu, "dw_up")):
            want = dd.T @ xd[a:b]
            err = ee.T @ xd[a:b].abs() + sum_error(b - a + 2, (dd.abs() + ee).T @ xd[a:b].abs())
            assert_within(got[e], want, rounded(want, err), what)


FP8_CASES = [("few", 128, 8, 0, "silu"), ("edges", 384, 136, 448, "silu"), ("large", 256, 72, 0, "gelu"),
             ("one_token", 1024, 200, 0, "silu"), ("none", 128, 64, 0, "silu")]


@pytest.mark.parametrize("case", FP8_CASES, ids=lambda c: "-".join(map(str, c)))
def test_gated_forward_fp8(case):
    """E4M3 products are exact in fp32 up to the sums: 448 * 448 needs 8 bits of significand. Each 128-element block
    is summed (128 additions), scaled (one rounding) and added (one), then the output scale multiplies."""
    counts, H, I, pitch, name = case
    g = torch.Generator().manual_seed(3)
    pk = packed(counts, H, payload="fp8", row_pitch=pitch)
    x = torch.randn(pk.rows, H, generator=g)
    x[: pk.P, :128] *= 100.0  # blocks of very different scales
    if pk.P:
        x[0] = 0.0            # an all-zero row: scale 0
    q, s = quantise_rows(x)
    q[pk.P:] = 0x7F           # NaN behind the last row
    s[pk.P:] = float("nan")
    buf = torch.full((pk.rows, pitch or H), 0x7F, dtype=torch.uint8)
    buf[:, :H] = q
    qg, sg = quantise_weights(torch.randn(8, I, H, generator=g) * H ** -0.5)
    qu, su = quantise_weights(torch.randn(8, I, H, generator=g) * H ** -0.5)
    d = pk.dev
    h, pre = pk.out(I), pk.out(2 * I)
    epl.experts_gated(pk.cfg, buf.to(d)[:, :H], pk.L, qg.to(d), qu.to(d), name, s.to(d), sg.to(d), su.to(d), h, pre)
    torch.cuda.synchronize()
    want, bound, wpre, pbound = gated_reference(pk, dequantise_rows(q[: pk.P], s[: pk.P]), dequantise_weights(qg, sg),
                                                dequantise_weights(qu, su), name)
    assert_within(h[: pk.P], want, bound, "h")
    assert_within(pre[: pk.P], wpre, pbound, "pre")
    pk.assert_untouched(h, "h")
    pk.assert_untouched(pre, "pre")


LINEAR_CASES = [  # counts, K, N, in pitch, out pitch, activation, bias, residual (own pitch), gap
    ("few", 8, 8, 0, 0, "none", False, False, 0),
    ("few", 72, 200, 80, 256, "silu", True, True, 0),
    ("one_token", 264, 512, 0, 0, "none", True, False, 0),
    ("edges", 136, 136, 0, 192, "gelu", True, True, 24),
    ("edges", 128, 64, 0, 0, "none", False, True, 0),
    ("one_expert", 104, 328, 0, 0, "relu", True, False, 0),
    ("none", 64, 64, 0, 0, "gelu", True, True, 0),
    ("large", 296, 192, 304, 256, "none", True, True, 0),
    ("large", 40, 1032, 0, 0, "silu", False, False, 0),
]


@pytest.mark.parametrize("case", LINEAR_CASES, ids=lambda c: "-".join(map(str, c)))
def test_linear_forward(case):
    counts, K, N, ip, op, name, has_bias, has_res, gap = case
    g = torch.Generator().manual_seed(4)
    pk = packed(counts, max(N, 8))
    a = pk.buffer(g, K, ip)
    w = weights(g, 8, N, K, pk.dev, N * K + gap if gap else 0)
    bias = torch.randn(8, N, generator=g).bfloat16().to(pk.dev) if has_bias else None
    res = pk.buffer(g, N, N + 16) if has_res else None
    out, pre = pk.out(N, op), pk.out(N)
    epl.experts_linear(pk.cfg, a, pk.L, w, bias, res, name, out=out, pre=pre)
    alone, none = epl.experts_linear(pk.cfg, a, pk.L, w, bias, res, name)
    torch.cuda.synchronize()
    assert none is None and torch.equal(alone[: pk.P], out[: pk.P])
    pk.assert_untouched(out, "out")
    pk.assert_untouched(pre, "pre")
    ad, wd = a.cpu().double(), w.cpu().double()
    for e, r0, r1 in pk.experts():
        v = ad[r0:r1] @ wd[e].T
        err = sum_error(K + 2, ad[r0:r1].abs() @ wd[e].abs().T)
        if has_bias:
            v = v + bias[e].cpu().double()
            err = err + FEW * (v.abs() + bias[e].cpu().double().abs())
        assert_within(pre[r0:r1], v, rounded(v, err), "pre")
        y = act(name, v)
        err = SLOPE * err + FEW * y.abs()
        if has_res:
            r = res[r0:r1].cpu().double()
            y = y + r
            err = err + FEW * (y.abs() + r.abs())
        assert_within(out[r0:r1], y, rounded(y, err), "out")


@pytest.mark.parametrize("case", LINEAR_CASES, ids=lambda c: "-".join(map(str, c)))
def test_linear_backward(case):
    counts, K, N, ip, op, name, has_bias, _, gap = case
    g = torch.Generator().manual_seed(5)
    pk = packed(counts, max(N, 8))
    a, dy = pk.buffer(g, K, ip), pk.buffer(g, N, op)
    pre = pk.buffer(g, N) if name != "none" else None
    w = weights(g, 8, N, K, pk.dev, N * K + gap if gap else 0)
    da = pk.out(K, ip)
    _, dw, db = epl.experts_linear_backward(pk.cfg, dy, a, pk.L, w, pre, name, need_dbias=has_bias, da=da)
    torch.cuda.synchronize()
    assert (db is not None) == has_bias
    pk.assert_untouched(da, "da")
    ad, wd, dyd = a.cpu().double(), w.cpu().double(), dy.cpu().double()
    for e, r0, r1 in pk.experts():
        if r0 == r1:
            assert not dw[e].any() and (db is None or not db[e].any())
            continue
        d = dyd[r0:r1]
        er = torch.zeros_like(d)
        sums = FEW * d.abs() * SLOPE
        if name != "none":
            d = d * act_grad(name, pre[r0:r1].cpu().double())
            er = rounded(d, sums)
        want = d @ wd[e]
        err = er @ wd[e].abs() + sum_error(N + 2, (d.abs() + er) @ wd[e].abs())
        assert_within(da[r0:r1], want, rounded(want, err), "da")
        want = d.T @ ad[r0:r1]
        err = er.T @ ad[r0:r1].abs() + sum_error(r1 - r0 + 2, (d.abs() + er).T @ ad[r0:r1].abs())
        assert_within(dw[e], want, rounded(want, err), "dw")
        if has_bias:
            want = d.sum(0)
            err = sums.sum(0) + sum_error(r1 - r0 + 2, d.abs().sum(0))
            assert_within(db[e], want, rounded(want, err), "dbias")


def test_linear_forward_fp8():
    counts, K, N = "edges", 256, 200
    g = torch.Generator().manual_seed(6)
    pk = packed(counts, K, payload="fp8")
    q, s = quantise_rows(torch.randn(pk.rows, K, generator=g))
    qw, sw = quantise_weights(torch.randn(8, N, K, generator=g))
    bias = torch.randn(8, N, generator=g).bfloat16()
    d = pk.dev
    out = pk.out(N)
    epl.experts_linear(pk.cfg, q.to(d), pk.L, qw.to(d), bias.to(d), None, "relu", s.to(d), sw.to(d), out=out)
    torch.cuda.synchronize()
    x, w = dequantise_rows(q, s), dequantise_weights(qw, sw)
    for e, r0, r1 in pk.experts():
        v = x[r0:r1] @ w[e].T + bias[e].double()
        err = sum_error(K + 4, x[r0:r1].abs() @ w[e].abs().T) + FEW * (v.abs() + bias[e].double().abs())
        y = v.clamp_min(0)
        assert_within(out[r0:r1], y, rounded(y, err), "out")
    pk.assert_untouched(out, "out")


def test_residual_in_place():
    g = torch.Generator().manual_seed(7)
    for counts, K, N in (("edges", 136, 264), ("one_token", 64, 72)):
        pk = packed(counts, N)
        a, w, res = pk.buffer(g, K), weights(g, 8, N, K, pk.dev), pk.buffer(g, N)
        want, _ = epl.experts_linear(pk.cfg, a, pk.L, w, residual=res)
        out = res.clone()
        epl.experts_linear(pk.cfg, a, pk.L, w, residual=out, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out[: pk.P], want[: pk.P])


def test_many_rows_take_the_large_tiles():
    """1024 rows an expert and more run on 256 x 256 tiles: odd features and ragged counts there too."""
    g = torch.Generator().manual_seed(8)
    rng = np.random.default_rng(8)
    counts = [1030, 1281, 777, 1200]
    pk = Packed(routing_of_counts(counts, 4, 2, rng), 4, 264, device())
    assert pk.rows // 4 >= 1024
    x, wg, wu = pk.buffer(g, 264), weights(g, 4, 152, 264, pk.dev), weights(g, 4, 152, 264, pk.dev)
    h, pre = pk.out(152), pk.out(304)
    epl.experts_gated(pk.cfg, x, pk.L, wg, wu, "silu", h=h, pre=pre)
    wd, bias, res = weights(g, 4, 264, 152, pk.dev), torch.randn(4, 264, generator=g).bfloat16().to(pk.dev), pk.buffer(g, 264)
    a = pk.buffer(g, 152)
    out = pk.out(264)
    epl.experts_linear(pk.cfg, a, pk.L, wd, bias, res, "none", out=out)
    torch.cuda.synchronize()
    want, bound, wpre, pbound = gated_reference(pk, x[: pk.P].cpu().double(), wg.cpu().double(), wu.cpu().double(), "silu")
    assert_within(h[: pk.P], want, bound, "h")
    assert_within(pre[: pk.P], wpre, pbound, "pre")
    ad, wd = a.cpu().double(), wd.cpu().double()
    for e, r0, r1 in pk.experts():
        b, r = bias[e].cpu().double(), res[r0:r1].cpu().double()
        y = ad[r0:r1] @ wd[e].T + b + r
        err = sum_error(152 + 2, ad[r0:r1].abs() @ wd[e].abs().T) + FEW * (y.abs() + b.abs() + r.abs())
        assert_within(out[r0:r1], y, rounded(y, err), "out")
    pk.assert_untouched(out, "out")


def test_fp8_many_rows():
    """256 rows an expert and more take the 128-row tiles; fewer the 64-row ones."""
    g = torch.Generator().manual_seed(10)
    rng = np.random.default_rng(10)
    pk = Packed(routing_of_counts([300, 270, 1, 510], 4, 1, rng), 4, 384, device(), payload="fp8")
    q, s = quantise_rows(torch.randn(pk.rows, 384, generator=g))
    qg, sg = quantise_weights(torch.randn(4, 136, 384, generator=g) * 384 ** -0.5)
    qu, su = quantise_weights(torch.randn(4, 136, 384, generator=g) * 384 ** -0.5)
    d = pk.dev
    h, pre = pk.out(136), pk.out(272)
    epl.experts_gated(pk.cfg, q.to(d), pk.L, qg.to(d), qu.to(d), "silu", s.to(d), sg.to(d), su.to(d), h, pre)
    torch.cuda.synchronize()
    want, bound, wpre, pbound = gated_reference(pk, dequantise_rows(q, s), dequantise_weights(qg, sg),
                                                dequantise_weights(qu, su), "silu")
    assert_within(h[: pk.P], want, bound, "h")
    assert_within(pre[: pk.P], wpre, pbound, "pre")


def test_offsets_that_hold_anything_stay_in_the_buffers():
    """expert_off is read on the device: whatever it holds, the rows read and written are the buffer's own."""
    g = torch.Generator().manual_seed(11)
    pk = packed("edges", 64)
    x, wg, wu = pk.buffer(g, 64), weights(g, 8, 64, 64, pk.dev), weights(g, 8, 64, 64, pk.dev)
    x.nan_to_num_(0.0)
    guard = torch.full((3 * pk.rows, 64), 77.0, dtype=torch.bfloat16, device=pk.dev)
    h = guard[pk.rows:2 * pk.rows]
    for off in ([-5] * 9, [2 ** 31 - 1] * 9, [0, 10 ** 9, 5, -7, 3, 2 ** 31 - 1, 0, 1, 10 ** 9], list(range(900, 0, -100))):
        pk.L.expert_off.copy_(torch.tensor(off, dtype=torch.int32))
        epl.experts_gated(pk.cfg, x, pk.L, wg, wu, h=h)
        dpre = torch.zeros(pk.rows, 128, dtype=torch.bfloat16, device=pk.dev)
        epl.experts_gated_backward(pk.cfg, x, dpre, x, pk.L, wg, wu, drecv=h)
        torch.cuda.synchronize()
        assert bool((guard[: pk.rows] == 77.0).all()) and bool((guard[2 * pk.rows:] == 77.0).all())


@pytest.mark.parametrize("E", [65, 200, 1024])
def test_many_experts_mostly_empty(E):
    """Row tiles are found 64 experts at a time: rows in the first and last expert of each group, none in most."""
    g = torch.Generator().manual_seed(E)
    rng = np.random.default_rng(E)
    counts = [0] * E
    for e in {0, 1, 63, 64, E - 1, E // 2, min(128, E - 1), min(191, E - 1)}:
        counts[e] = int(rng.integers(1, 150))
    pk = Packed(routing_of_counts(counts, E, 2, rng), E, 64, device())
    x, wg, wu = pk.buffer(g, 64), weights(g, E, 72, 64, pk.dev), weights(g, E, 72, 64, pk.dev)
    h, pre = epl.experts_gated(pk.cfg, x, pk.L, wg, wu, keep_pre=True)
    dh = pk.buffer(g, 72)
    dx, dwg, dwu = epl.experts_gated_backward(pk.cfg, dh, pre, x, pk.L, wg, wu)
    torch.cuda.synchronize()
    want, bound, wpre, pbound = gated_reference(pk, x[: pk.P].cpu().double(), wg.cpu().double(), wu.cpu().double(), "silu")
    assert_within(h[: pk.P], want, bound, "h")
    assert_within(pre[: pk.P], wpre, pbound, "pre")
    p, d, xd = pre.cpu().double(), dh.cpu().double(), x.cpu().double()
    for e, a, b in pk.experts():
        if a == b:
            assert not dwg[e].any() and not dwu[e].any(), e
            continue
        gg, u = p[a:b, :72], p[a:b, 72:]
        dg, du = d[a:b] * u * act_grad("silu", gg), d[a:b] * act("silu", gg)
        eg, eu = rounded(dg, FEW * (d[a:b] * u).abs() * SLOPE), rounded(du, FEW * (d[a:b] * gg).abs())
        w = (wg[e].cpu().double(), wu[e].cpu().double())
        want = dg @ w[0] + du @ w[1]
        err = eg @ w[0].abs() + eu @ w[1].abs() + sum_error(146, (dg.abs() + eg) @ w[0].abs() + (du.abs() + eu) @ w[1].abs())
        assert_within(dx[a:b], want, rounded(want, err), "drecv")
        want = dg.T @ xd[a:b]
        err = eg.T @ xd[a:b].abs() + sum_error(b - a + 2, (dg.abs() + eg).T @ xd[a:b].abs())
        assert_within(dwg[e], want, rounded(want, err), "dw_gate")


def test_no_tokens():
    """No rows at all: nothing to do forward, zero gradients of the weights backward."""
    dev = device()
    cfg = epl.config(2, 4, 2, 64, 0)
    L = epl.layout(cfg, torch.empty(0, 2, dtype=torch.int32, device=dev))
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=dev)
    g = torch.Generator().manual_seed(1)
    w = weights(g, 4, 32, 64, dev)
    h, pre = epl.experts_gated(cfg, x, L, w, w, keep_pre=True)
    _, dwg, dwu = epl.experts_gated_backward(cfg, h, pre, x, L, w, w)
    y, _ = epl.experts_linear(cfg, x, L, w)
    _, dw, db = epl.experts_linear_backward(cfg, y, x, L, w, need_dbias=True)
    torch.cuda.synchronize()
    assert not dwg.any() and not dwu.any() and not dw.any() and not db.any()


def test_refused_tensors():
    """What the binding refuses before a launch: overlapping matrices, short buffers, wrong pitches and types."""
    g = torch.Generator().manual_seed(2)
    pk = packed("few", 64)
    x, w = pk.buffer(g, 64), weights(g, 8, 32, 64, pk.dev)
    with pytest.raises(ValueError, match="overlap"):
        epl.experts_gated(pk.cfg, x, pk.L, w[:1].expand(8, 32, 64), w[:1].expand(8, 32, 64))
    with pytest.raises(ValueError, match="rows"):
        epl.experts_gated(pk.cfg, x[:-1], pk.L, w, w)
    with pytest.raises(ValueError, match="apart"):
        epl.experts_gated(pk.cfg, pk.buffer(g, 64, 128), pk.L, w, w)
    with pytest.raises(ValueError, match="contiguous"):
        epl.experts_linear(pk.cfg, x, pk.L, w.transpose(1, 2))
    with pytest.raises(ValueError):
        epl.experts_linear(pk.cfg, x.float(), pk.L, w)
    with pytest.raises(epl.EplError, match="ALIGN"):
        epl.experts_linear(pk.cfg, x, pk.L, w, bias=torch.zeros(8 * 32 + 1, dtype=torch.bfloat16, device=pk.dev)[1:].view(8, 32))
    with pytest.raises(epl.EplError, match="INVALID"):
        epl.experts_gated_backward(pk.cfg, pk.buffer(g, 32), pk.buffer(g, 64), x, pk.L, w, w, drecv=x)


@pytest.mark.parametrize("counts", [[3, 0], [20, 9]], ids=["few", "tiles"])
def test_largest_feature_counts(counts):
    """EPL_MAX_HIDDEN features on either side of a product. The inputs are small integers, mostly zero, so fp32 sums are
    exact and a result is the integer, rounded once."""
    N, E = 1 << 20, 2
    g = torch.Generator(device=device()).manual_seed(12)
    rng = np.random.default_rng(12)
    pk = Packed(routing_of_counts(counts, E, 1, rng), E, N, device())

    def small(*shape):
        return torch.randint(-2, 3, shape, generator=g, device=pk.dev).bfloat16()

    # A reduction over 2^20: sums stay below 2^22.
    x, wg, wu = small(pk.rows, N), small(E, 8, N), small(E, 8, N)
    _, pre = epl.experts_gated(pk.cfg, x, pk.L, wg, wu, "none", keep_pre=True)
    # 2^20 results, and gradients that reduce over them.
    a, w, bias = small(pk.rows, 8), small(E, N, 8), small(E, N)
    out, _ = epl.experts_linear(pk.cfg, a, pk.L, w, bias)
    dy = small(pk.rows, N)
    da, dw, db = epl.experts_linear_backward(pk.cfg, dy, a, pk.L, w, need_dbias=True)
    torch.cuda.synchronize()
    for e, r0, r1 in pk.experts():
        xs, ws, d = x[r0:r1].float(), w[e].float(), dy[r0:r1].float()
        both = torch.cat([wg[e], wu[e]]).float()
        for r in range(r1 - r0):  # integers, summed in 64 bits
            want = (both.double() * xs[r].double()).sum(1)
            assert torch.equal(pre[r0 + r], want.float().bfloat16()), (e, r)
            want = (d[r].double()[:, None] * ws.double()).sum(0)
            assert torch.equal(da[r0 + r], want.float().bfloat16()), (e, r)
            want = (ws.double() * a[r0 + r].double()).sum(1) + bias[e].double()
            assert torch.equal(out[r0 + r], want.float().bfloat16()), (e, r)
        want = torch.zeros(N, 8, dtype=torch.float64, device=pk.dev)
        for r in range(r0, r1):
            want += dy[r].double()[:, None] * a[r].double()[None]
        assert torch.equal(dw[e], want.float().bfloat16()), e
        assert torch.equal(db[e], dy[r0:r1].double().sum(0).float().bfloat16()), e
