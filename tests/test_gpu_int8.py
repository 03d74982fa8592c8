"""Rows in int8 (epl_dispatch_int8, epl_quantize_rows) bit for bit against the definition in 64 bits, and the experts'
products of them against exact integer sums, at the sizes where a piece, a pass, a tile or a segment ends.

Bounds of the products: the sum is exact; its conversion and the two scales are three roundings (2^-24 each), the bias and
the residual one more each; then as in products_util."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import FEW, SLOPE, Packed, act, assert_within, rounded, routing_of_counts

pytestmark = pytest.mark.gpu

ONE = 2.0 ** -24
INF = float("inf")


def quantised(x: torch.Tensor):
    """Rows of bf16 on the host -> (int8 rows, fp32 scales) by the definition, in 64 bits: 127 |x| / max|x| is exact where
    it is a half, and otherwise further from one than its rounding."""
    a = x.double()
    top = a.abs().amax(1, keepdim=True)
    bad = ~torch.isfinite(a).all(1, keepdim=True)
    live = (top > 0) & ~bad
    r = torch.where(live, 127 * a.abs() / torch.where(live, top, 1.0), 0.0)
    down = torch.floor(r)
    up = (r - down > 0.5) | ((r - down == 0.5) & (down % 2 == 1))
    q = ((down + up) * torch.where(a < 0, -1.0, 1.0)).to(torch.int8)
    s = x.abs().amax(1).float() / torch.tensor(127.0)
    return q, torch.where(bad[:, 0], float("nan"), s)


def assert_rows(q, s, x, what):
    want, scale = quantised(x.cpu())
    assert torch.equal(q.cpu(), want), what
    assert torch.equal(torch.nan_to_num(s.cpu(), -1.0), torch.nan_to_num(scale, -1.0)), what


def int8_out(pk, width, pitch=0):
    return torch.full((pk.rows, pitch or width), 77, dtype=torch.int8, device=pk.dev)[:, :width]


def assert_behind(pk, q, s, what):
    pk.assert_untouched(q, what)
    assert bool((s[pk.P:] == 77.0).all()), what + ": scales behind the last were written"


# ---------------------------------------------------------------- rows
@pytest.mark.parametrize("K", [16, 32, 240, 256, 272, 512, 528, 1008, 1024, 1040, 2048, 2064, 4080, 4096, 4112, 7168, 8192, 8208,
                               16384, 16400, 32768, 32784, 70000])
def test_quantize_weights_at_the_ends_of_pieces_and_passes(K):
    g = torch.Generator().manual_seed(K)
    w = (torch.randn(3, 5, K, generator=g) * torch.exp(torch.randn(3, 5, 1, generator=g) * 3)).bfloat16()
    w[0, 0, -1] = 1000.0  # the maximum in the last place
    w[0, 1, 0] = -1000.0
    w[0, 2] = 0.0
    w[0, 3, :-1] = 0.0
    q, s = epl.quantize_weights(w.to(device()))
    torch.cuda.synchronize()
    assert_rows(q.view(15, K), s.view(-1), w.view(15, K), "K = %d" % K)
    assert not q[0, 2].any() and float(s[0, 2]) == 0.0


def test_every_mantissa_against_every_other():
    """A row for each mantissa of the maximum and each of four sizes: all 128 mantissas at 11 exponents from it down, both
    signs. Among them are all halves that there are."""
    rows = []
    for e in (0, 100, -100, -112):
        for top in range(128, 256):
            m = torch.arange(128, 256, dtype=torch.float64)
            v = torch.cat([torch.ldexp(m, torch.tensor(e - 7 - gap)) for gap in range(11)])
            limit = np.ldexp(float(top), e - 7)
            v = torch.where(v <= limit, v, 0.0)
            rows.append(torch.cat([v, -v, torch.full((16,), limit, dtype=torch.float64)]))
    x = torch.stack(rows)
    assert bool((x.bfloat16().double() == x).all())  # every value is a bf16 one
    q, s = epl.quantize_weights(x.bfloat16().view(1, *x.shape).to(device()))
    torch.cuda.synchronize()
    assert_rows(q[0], s[0], x.bfloat16(), "mantissas")


def test_subnormals_and_the_largest():
    least, last = 2.0 ** -133, float(torch.finfo(torch.bfloat16).max)
    x = torch.zeros(6, 32, dtype=torch.bfloat16)
    x[0, 0], x[0, 1] = least, -least
    x[1, :3] = torch.tensor([127 * least, 64 * least, least])
    x[2, :3] = torch.tensor([2.0 ** -126, 2.0 ** -127, -2.0 ** -130])
    x[3, :4] = torch.tensor([last, -last / 2, last / 255, 1.0])
    x[4, :3] = torch.tensor([-last, 2.0 ** 100, least])
    x[5, :3] = torch.tensor([2.0 ** -100, 2.0 ** -101, 2.0 ** -108])
    q, s = epl.quantize_weights(x[None].to(device()))
    torch.cuda.synchronize()
    assert_rows(q[0], s[0], x, "subnormals")


@pytest.mark.parametrize("K", [16, 384, 768, 2048, 9216])
def test_infinities_and_nan(K):
    x = torch.randn(5, K, generator=torch.Generator().manual_seed(1)).bfloat16()
    x[0, 3], x[1, -1], x[2, 0], x[3, 5] = INF, -INF, float("nan"), 0.0
    x[3].view(torch.int16)[7] = -1  # a negative NaN with every bit set
    q, s = epl.quantize_weights(x[None].to(device()))
    torch.cuda.synchronize()
    assert_rows(q[0], s[0], x, "not finite")
    assert bool(torch.isnan(s[0, :4]).all()) and not q[0, :4].any() and q[0, 4].any()


@pytest.mark.parametrize("T,k,K,pitch,qpitch", [(1, 1, 16, 0, 0), (9, 2, 784, 800, 832), (3, 4, 4112, 0, 0),
                                                (700, 2, 64, 72, 0), (333, 3, 400, 0, 448), (40, 8, 16400, 0, 16448), (2100, 1, 2048, 0, 0)])
def test_quantize_packed_rows(T, k, K, pitch, qpitch):
    g = torch.Generator().manual_seed(K)
    rng = np.random.default_rng(T)
    idx = rng.integers(-1, 9, (T, k)).astype(np.int32)
    idx[0] = 3
    pk = Packed(idx, 8, 64, device())
    a = pk.buffer(g, K, pitch, std=3.0)
    q, s = int8_out(pk, K, qpitch), torch.full((pk.rows,), 77.0, device=pk.dev)
    epl.quantize_rows(pk.cfg, a, pk.L, q=q, q_scale=s)
    new, new_s = epl.quantize_rows(pk.cfg, a, pk.L)
    torch.cuda.synchronize()
    assert_rows(q[: pk.P], s[: pk.P], a[: pk.P], "rows")
    assert torch.equal(new[: pk.P], q[: pk.P]) and torch.equal(new_s[: pk.P], s[: pk.P])
    assert_behind(pk, q, s, "q")


DISPATCH = [(1, 8, 1, 1, 16, 0), (2, 8, 2, 9, 272, 320), (4, 16, 8, 33, 1024, 0), (4, 64, 8, 16, 7168, 7232),
            (1, 40, 12, 21, 2064, 0), (2, 64, 32, 5, 528, 576), (1, 8, 3, 7, 9232, 0), (2, 8, 2, 3, 40000, 0),
            (8, 32, 4, 260, 2048, 0), (1, 8, 3, 700, 4112, 0), (1, 4, 3, 0, 64, 0)]


def choices(R, E, k, Tr, rng):
    idx = rng.integers(-1, E + 1, (R * Tr, k)).astype(np.int32)  # some invalid, some twice
    if Tr > 2:
        idx[-2:] = -1
    return idx


@pytest.mark.parametrize("R,E,k,Tr,H,pitch", DISPATCH)
@pytest.mark.parametrize("weighted", [False, True])
def test_dispatch_int8(R, E, k, Tr, H, pitch, weighted):
    dev = device()
    g = torch.Generator().manual_seed(H + k)
    idx = choices(R, E, k, Tr, np.random.default_rng(k))
    if Tr == 0:
        cfg = epl.config(R, E, k, H, 0)
        epl.dispatch_int8(cfg, torch.zeros(1, H, dtype=torch.bfloat16, device=dev), epl.alloc_layout(cfg, dev))
        torch.cuda.synchronize()
        return
    pk = Packed(idx, E, H, dev, R=R, row_pitch=pitch)
    T = R * Tr
    x = (torch.randn(T, H, generator=g) * torch.exp(torch.randn(T, 1, generator=g))).bfloat16()
    x[0] = 0.0
    w = torch.randn(T, k, generator=g)
    w[torch.from_numpy((idx < 0) | (idx >= E))] = float("nan")  # not looked at
    q, s = int8_out(pk, H, pitch), torch.full((pk.rows,), 77.0, device=dev)
    epl.dispatch_int8(pk.cfg, x.to(dev), pk.L, topk_w=w.to(dev) if weighted else None, recv=q, recv_scale=s)
    torch.cuda.synchronize()
    row = pk.L.pair_row.cpu().long()
    tok, j = (row >= 0).nonzero(as_tuple=True)
    want, scale = quantised(x)
    assert torch.equal(q.cpu()[row[tok, j]], want[tok])
    scale = scale[tok] * w[tok, j] if weighted else scale[tok]
    assert torch.equal(s.cpu()[row[tok, j]], scale)
    assert_behind(pk, q, s, "recv")


# ---------------------------------------------------------------- products
COUNTS = {
    "one_token": [0, 0, 1, 0, 1, 0, 0, 1],
    "sixteen": [4, 0, 1, 2, 0, 5, 1, 3],
    "few": [3, 0, 1, 2, 0, 5, 16, 17],
    "edges": [127, 128, 129, 0, 1, 64, 255, 31],
    "one_expert": [0, 0, 0, 700, 0, 0, 0, 0],
    "none": [0, 0, 0, 0, 0, 0, 0, 0],
    "large": [513, 256, 300, 1, 0, 257, 640, 90],
    "many": [1500, 1024, 0, 1, 2000, 257, 1300, 2200],  # 1024 rows an expert and more: the largest tiles
}


def packed(counts, H, k=2, seed=0, **kw):
    idx = routing_of_counts(COUNTS[counts], 8, k, np.random.default_rng(seed))
    if counts not in ("one_token", "sixteen"):
        idx = np.concatenate([idx, np.full((3, k), -1, np.int32)])  # padded tokens
    return Packed(idx, 8, H, device(), **kw)


def int8_rows(pk, g, K, pitch=0):
    """Random int8 rows (-128 among them) with NaN scales behind the last one and 99 in the gaps."""
    b = torch.full((pk.rows, pitch or K), 99, dtype=torch.int8)
    b[: pk.P, :K] = torch.randint(-128, 128, (pk.P, K), generator=g, dtype=torch.int8)
    s = torch.full((pk.rows,), float("nan"))
    s[: pk.P] = torch.exp(torch.randn(pk.P, generator=g)) * 0.02
    return b.to(pk.dev)[:, :K], s.to(pk.dev)


def int8_matrices(g, N, K, dev, gap=0):
    b = torch.full((8, N * K + gap), 99, dtype=torch.int8)
    b[:, : N * K] = torch.randint(-128, 128, (8, N * K), generator=g, dtype=torch.int8)
    s = torch.exp(torch.randn(8, N, generator=g)) * K ** -0.5 * 0.02
    return b.to(dev).as_strided((8, N, K), (N * K + gap, K, 1)), s.to(dev)


def product(x, xs, w, ws):
    """The scaled product and its error bound."""
    v = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()[None]
    return v, 4 * ONE * v.abs()


GATED = [  # counts, H, I, pitch, activation, gap between matrices, halves of one tensor
    ("one_token", 512, 264, 0, "silu", 0, False),
    ("sixteen", 16, 8, 0, "silu", 0, False),
    ("sixteen", 208, 72, 256, "gelu", 0, True),
    ("sixteen", 2064, 40, 0, "relu", 16, False),
    ("few", 16, 8, 0, "silu", 0, False),
    ("few", 208, 72, 256, "gelu", 0, True),
    ("edges", 144, 136, 192, "silu", 64, False),
    ("edges", 64, 128, 0, "relu", 0, True),
    ("one_expert", 336, 104, 0, "none", 0, False),
    ("none", 64, 64, 0, "silu", 0, False),
    ("large", 192, 296, 256, "silu", 0, True),
    ("large", 1040, 40, 0, "gelu", 16, False),
    ("many", 16, 8, 0, "silu", 0, False),
    ("many", 656, 264, 704, "gelu", 32, False),
    ("many", 384, 520, 0, "silu", 0, True),
]


@pytest.mark.parametrize("case", GATED, ids=lambda c: "-".join(map(str, c)))
def test_gated(case):
    counts, H, I, pitch, name, gap, halves = case
    g = torch.Generator().manual_seed(1)
    pk = packed(counts, H, row_pitch=pitch)
    x, xs = int8_rows(pk, g, H, pitch)
    if halves:
        both, s = int8_matrices(g, 2 * I, H, pk.dev)
        wg, wu, gs, us = both[:, :I], both[:, I:], s[:, :I].contiguous(), s[:, I:].contiguous()
    else:
        (wg, gs), (wu, us) = int8_matrices(g, I, H, pk.dev, gap), int8_matrices(g, I, H, pk.dev, gap)
    h = pk.out(I)
    epl.experts_gated_int8(pk.cfg, x, xs, pk.L, wg, gs, wu, us, name, h=h)
    new = epl.experts_gated_int8(pk.cfg, x, xs, pk.L, wg, gs, wu, us, name)
    torch.cuda.synchronize()
    assert torch.equal(new[: pk.P], h[: pk.P])
    pk.assert_untouched(h, "h")
    for e, a, b in pk.experts():
        if a == b:
            continue
        v, dv = product(x[a:b].cpu(), xs[a:b].cpu(), wg[e].cpu(), gs[e].cpu())
        u, du = product(x[a:b].cpu(), xs[a:b].cpu(), wu[e].cpu(), us[e].cpu())
        r = act(name, v)
        err = SLOPE * dv * (u.abs() + du) + (r.abs() + FEW) * du + FEW * (r * u).abs()
        assert_within(h[a:b], r * u, rounded(r * u, err), "h of expert %d" % e)


LINEAR = [  # counts, K, N, in pitch, out pitch, activation, bias, residual, gap
    ("one_token", 768, 520, 0, 0, "none", False, False, 0),
    ("sixteen", 16, 8, 0, 0, "none", False, False, 0),
    ("sixteen", 208, 72, 256, 80, "gelu", True, True, 16),
    ("few", 16, 8, 32, 0, "silu", True, False, 0),
    ("edges", 144, 136, 0, 192, "none", True, True, 64),
    ("edges", 64, 264, 0, 0, "relu", False, True, 0),
    ("one_expert", 336, 104, 0, 0, "gelu", True, False, 0),
    ("none", 64, 64, 0, 0, "none", True, False, 0),
    ("large", 1040, 40, 1056, 64, "silu", True, True, 0),
    ("large", 192, 520, 0, 0, "none", False, False, 16),
    ("many", 16, 8, 0, 0, "none", True, True, 0),
    ("many", 656, 520, 672, 576, "gelu", True, True, 0),
    ("many", 384, 264, 0, 0, "none", False, False, 0),
]


@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(map(str, c)))
def test_linear(case):
    counts, K, N, ip, op, name, with_bias, with_res, gap = case
    g = torch.Generator().manual_seed(2)
    pk = packed(counts, 64)
    x, xs = int8_rows(pk, g, K, ip)
    w, ws = int8_matrices(g, N, K, pk.dev, gap)
    bias = torch.randn(8, N, generator=g).bfloat16().to(pk.dev) if with_bias else None
    res = pk.buffer(g, N, N + 8) if with_res else None
    out = pk.out(N, op)
    epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, bias, res, name, out=out)
    same = out.clone() if res is None else res.clone()
    epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, bias, None if res is None else same, name, out=same)  # in place
    torch.cuda.synchronize()
    assert torch.equal(same[: pk.P], out[: pk.P])
    pk.assert_untouched(out, "out")
    for e, a, b in pk.experts():
        if a == b:
            continue
        v, dv = product(x[a:b].cpu(), xs[a:b].cpu(), w[e].cpu(), ws[e].cpu())
        if with_bias:
            v = v + bias[e].cpu().double()
            dv = dv + ONE * (v.abs() + dv)
        r = act(name, v)
        err = SLOPE * dv + FEW * r.abs()
        if with_res:
            r = r + res[a:b].cpu().double()
            err = err + ONE * (r.abs() + err)
        assert_within(out[a:b], r, rounded(r, err), "out of expert %d" % e)


@pytest.mark.parametrize("rows", [1, 16, 40, 1100])
def test_the_longest_sums_are_exact(rows):
    """-128 * -128 over as many features as there can be is 2^31 - 262144; one product less is that minus 16384. With
    scales of 2^-31 and one, and 1 - 2^-13 and 1 - 2^-13 - 2^-17 in 32 bits, bf16 rounds both to one: the difference is
    looked at with a bias of minus one."""
    K = epl.MAX_INT8_FEATURES
    dev = device()
    pk = Packed(np.zeros((rows, 1), np.int32), 1, 64, dev)
    x = torch.full((rows, K), -128, dtype=torch.int8, device=dev)
    xs = torch.full((rows,), 2.0 ** -31, device=dev)
    w = torch.full((1, 16, K), -128, dtype=torch.int8, device=dev)
    w[0, 1, 70000] = 0
    w[0, 2] = 127
    out = epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, torch.ones(1, 16, device=dev),
                                  bias=torch.full((1, 16), -1.0, dtype=torch.bfloat16, device=dev))
    torch.cuda.synchronize()
    full = 16384 * K * 2.0 ** -31
    want = torch.full((16,), full - 1, dtype=torch.float64)
    want[1] = full - 2.0 ** -17 - 1
    want[2] = -128 * 127 * K * 2.0 ** -31 - 1
    assert torch.equal(out.cpu(), want.bfloat16().expand(rows, 16))


def test_a_row_that_was_not_finite():
    """Its products are NaN, the other rows' are not."""
    dev = device()
    g = torch.Generator().manual_seed(3)
    for rows in (9, 300):
        pk = Packed(np.zeros((rows, 1), np.int32), 1, 64, dev)
        x = torch.randn(rows, 64, generator=g).bfloat16().to(dev)
        x[2, 5] = INF
        q, s = epl.dispatch_int8(pk.cfg, x, pk.L)
        w, ws = epl.quantize_weights(torch.randn(1, 64, 64, generator=g).bfloat16().to(dev))
        h = epl.experts_gated_int8(pk.cfg, q, s, pk.L, w, ws, w, ws)
        y = epl.experts_linear_int8(pk.cfg, *epl.quantize_rows(pk.cfg, h, pk.L), pk.L, w, ws)
        torch.cuda.synchronize()
        bad = torch.zeros(rows, dtype=torch.bool, device=dev)
        bad[2] = True
        for t in (h, y):
            assert torch.equal(torch.isnan(t).all(1), bad) and torch.equal(torch.isnan(t).any(1), bad)


def test_the_largest_and_the_smallest_rows():
    """Rows near fp32's ends, whose sums times the row's scale alone would leave them: the product with the weights' small
    (large) scales is well inside."""
    dev = device()
    g = torch.Generator().manual_seed(4)
    for rows in (9, 40, 700, 2400):
        pk = Packed(np.zeros((rows, 1), np.int32), 1, 64, dev)
        for size, ws in ((2.0 ** 127, 2.0 ** -40), (2.0 ** -120, 2.0 ** 30)):
            x = (torch.randn(rows, 64, generator=g).clamp(-1.9, 1.9).double() * size).bfloat16()
            q, s = epl.dispatch_int8(pk.cfg, x.to(dev), pk.L)
            w = torch.randint(-127, 128, (1, 16, 64), generator=g, dtype=torch.int8)
            out = epl.experts_linear_int8(pk.cfg, q, s, pk.L, w.to(dev), torch.full((1, 16), ws, device=dev))
            h = epl.experts_gated_int8(pk.cfg, q, s, pk.L, w.to(dev), torch.full((1, 16), ws, device=dev), w.to(dev),
                                       torch.full((1, 16), 2.0 ** -100 * ws if size > 1 else ws, device=dev), "none")
            torch.cuda.synchronize()
            want = (q.cpu().double() @ w[0].double().T) * ws * s.cpu().double()[:, None]
            assert_within(out, want, rounded(want, 4 * ONE * want.abs()), "out")
            if size > 1:
                both = want * want * 2.0 ** -100
                assert_within(h, both, rounded(both, 10 * ONE * both.abs()), "h")


# ---------------------------------------------------------------- the layer as it is used
class Layer:
    """Router, int8 dispatch, gated product, int8 rows of it, the way down, combine."""

    def __init__(self, R=2, E=16, k=4, Tr=40, H=128, I=192, pitch=192, seed=0, pad=3):
        g = torch.Generator().manual_seed(seed)
        self.cfg = epl.config(R, E, k, H, Tr, "bf16", pitch)
        T = R * Tr
        logits = torch.randn(T, E, generator=g)
        logits.view(R, Tr, E)[:, Tr - pad:] = -INF
        bf = lambda *shape, std=1.0: (torch.randn(*shape, generator=g) * std).bfloat16()
        self.host = dict(logits=logits, x=bf(T, H), wg=bf(E, I, H, std=H ** -0.5), wu=bf(E, I, H, std=H ** -0.5),
                         wd=bf(E, H, I, std=I ** -0.5), b=bf(E, H, std=0.2))
        self.d = {n: t.to(device()) for n, t in self.host.items()}
        self.w = {n: epl.quantize_weights(self.d[n]) for n in ("wg", "wu", "wd")}

    def forward(self, before=False):
        """before: the gate weights go into the dispatched rows' scales, and combine adds with ones."""
        cfg, d = self.cfg, self.d
        idx, w = epl.route(cfg, d["logits"])
        L = epl.layout(cfg, idx)
        q, s = epl.dispatch_int8(cfg, d["x"], L, topk_w=w if before else None)
        h = epl.experts_gated_int8(cfg, q, s, L, *self.w["wg"], *self.w["wu"])
        y = epl.experts_linear_int8(cfg, *epl.quantize_rows(cfg, h, L), L, *self.w["wd"], bias=d["b"])
        return epl.combine(cfg, y, torch.ones_like(w) if before else w, L), (idx, w)

    def reference(self, idx, w, before):
        """The same in 64 bits: int8 values and scales by the definition, of rows and of weights."""
        def values(t):
            q, s = quantised(t.reshape(-1, t.shape[-1]))
            return (q.double() * s.double()[:, None]).view(t.shape)
        x, wg, wu, wd = (values(self.host[n]) for n in ("x", "wg", "wu", "wd"))
        out = torch.zeros_like(x)
        for j in range(idx.shape[1]):
            for e in range(self.cfg.num_experts):
                t = (idx[:, j] == e).nonzero()[:, 0]
                if not t.numel():
                    continue
                wt = w[t, j, None].double()
                xe = x[t] * wt if before else x[t]
                h = torch.nn.functional.silu(xe @ wg[e].T) * (xe @ wu[e].T)
                y = values(h.bfloat16()) @ wd[e].T + self.host["b"][e].double()
                out.index_add_(0, t, y if before else y * wt)
        return out


@pytest.mark.parametrize("before", [False, True])
@pytest.mark.parametrize("shape", [dict(), dict(R=1, E=8, k=2, Tr=1, H=64, I=64, pitch=0, pad=0),
                                   dict(R=4, E=32, k=8, Tr=130, H=272, I=144, pitch=320, pad=7, seed=3),
                                   dict(R=2, E=8, k=3, Tr=17, H=128, I=128, pitch=0, pad=17, seed=4)],
                         ids=["small", "one_token", "odd", "all_padding"])
def test_layer(shape, before):
    layer = Layer(**shape)
    out, (idx, w) = layer.forward(before)
    torch.cuda.synchronize()
    want = layer.reference(idx.cpu().long(), w.cpu(), before)
    if not want.any():
        assert not out.any()
        return
    # h, y and out are rounded to bf16 (2^-8 of their norms each, at most). A value of h next to a rounding border of bf16
    # or of int8 may fall to the other side: then it is off by one step of bf16 (2^-7 of it) or by max / 127 of its row. The
    # kernels' h is within 2^-20 of the reference's before rounding, so this happens to a value in 2^-20 / 2^-8 (bf16) or
    # less than one in 2^-20 * 127 (int8): some tens of values at most of some 10^5, whose squares add nothing to the norm
    # (127^-2 * 16 * 2^-12 against 2^-16).
    assert float((out.cpu().double() - want).norm() / want.norm()) <= 3 * 2.0 ** -8


def test_no_tokens():
    dev = device()
    cfg = epl.config(2, 8, 2, 64, 0)
    L = epl.layout(cfg, torch.zeros(0, 2, dtype=torch.int32, device=dev))
    w, ws = epl.quantize_weights(torch.ones(8, 64, 64, dtype=torch.bfloat16, device=dev))
    q, s = epl.dispatch_int8(cfg, torch.zeros(0, 64, dtype=torch.bfloat16, device=dev), L)
    h = epl.experts_gated_int8(cfg, q, s, L, w, ws, w, ws)
    y = epl.experts_linear_int8(cfg, *epl.quantize_rows(cfg, h, L), L, w, ws)
    torch.cuda.synchronize()
    assert y.shape[1] == 64
    q, s = epl.quantize_weights(torch.ones(0, 64, 64, dtype=torch.bfloat16, device=dev))
    assert q.shape == (0, 64, 64) and s.shape == (0, 64)


def test_what_a_layout_of_all_padding_leaves():
    dev = device()
    pk = Packed(np.full((9, 2), -1, np.int32), 8, 64, dev, row_pitch=128)
    q, s = int8_out(pk, 64, 128), torch.full((18,), 77.0, device=dev)
    epl.dispatch_int8(pk.cfg, torch.ones(9, 64, dtype=torch.bfloat16, device=dev), pk.L, recv=q, recv_scale=s)
    epl.quantize_rows(pk.cfg, pk.out(64), pk.L, q=q, q_scale=s)
    torch.cuda.synchronize()
    assert_behind(pk, q, s, "padding")


def test_another_stream_and_a_captured_graph():
    layer = Layer(seed=8)
    torch.cuda.synchronize()
    want, _ = layer.forward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again, _ = layer.forward()
    s.synchronize()
    assert torch.equal(want, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = layer.forward()
        before, _ = layer.forward(True)
    for seed in range(4):
        other = Layer(seed=20 + seed, pad=seed)
        for n, t in layer.d.items():
            t.copy_(other.d[n])
        for n, pair in layer.w.items():
            for a, b in zip(pair, other.w[n]):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other.forward()[0]) and torch.equal(before, other.forward(True)[0]), seed
        torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """int8 rows and matrices past 4 GiB: the last ones against the same alone."""
    dev = device()
    g = torch.Generator().manual_seed(9)
    E, K, N = 80, 8192, 8192  # 5.4 GB of matrices
    counts = [0] * E
    counts[0], counts[-1] = 5, 40
    pk = Packed(routing_of_counts(counts, E, 1, np.random.default_rng(1)), E, 64, dev)
    w = torch.empty(E, N, K, dtype=torch.int8, device=dev)
    ws = torch.ones(E, N, device=dev)
    w[-1], ws[-1] = (t[0] for t in epl.quantize_weights(torch.randn(1, N, K, generator=g).bfloat16().to(dev)))
    w[0], ws[0] = w[-1], ws[-1]
    a = torch.randint(-127, 128, (45, K), generator=g, dtype=torch.int8).to(dev)
    xs = torch.full((45,), 0.01, device=dev)
    out = epl.experts_linear_int8(pk.cfg, a, xs, pk.L, w, ws)
    one = Packed(np.zeros((45, 1), np.int32), 1, 64, dev)
    want = epl.experts_linear_int8(one.cfg, a, xs, one.L, w[-1:].contiguous(), ws[-1:].contiguous())
    torch.cuda.synchronize()
    assert torch.equal(out[:45], want[:45])
    del w
    torch.cuda.empty_cache()
    rows, pitch = 140000, 32768  # 4.6 GB of int8 rows, 9.2 GB of bf16 ones
    idx = np.zeros((rows, 1), np.int32)
    idx[-100:] = 1
    far = Packed(idx, 2, 64, dev, row_pitch=pitch)
    x = torch.zeros(rows, 64, dtype=torch.bfloat16, device=dev)
    x[-100:] = torch.randn(100, 64, generator=g).bfloat16().to(dev)
    recv = torch.empty(rows, pitch, dtype=torch.int8, device=dev)[:, :64]
    q, s = epl.dispatch_int8(far.cfg, x, far.L, recv=recv)
    torch.cuda.synchronize()
    assert not q[:-100].any() and not s[:-100].any()
    assert_rows(q[-100:], s[-100:], x[-100:], "far rows")
    wide = torch.empty(rows, pitch, dtype=torch.bfloat16, device=dev)[:, :64]
    wide.copy_(x)
    recv.zero_()
    q2, s2 = epl.quantize_rows(far.cfg, wide, far.L, q=recv)
    torch.cuda.synchronize()
    assert_rows(q2[-100:], s2[-100:], x[-100:], "far rows")
    w, ws = epl.quantize_weights(torch.randn(2, 64, 64, generator=g).bfloat16().to(dev))
    h = epl.experts_gated_int8(far.cfg, recv, s2, far.L, w, ws, w, ws)
    near = Packed(np.zeros((100, 1), np.int32), 1, 64, dev)
    want = epl.experts_gated_int8(near.cfg, q2[-100:].contiguous(), s2[-100:].contiguous(), near.L, w[1:].contiguous(),
                                  ws[1:].contiguous(), w[1:].contiguous(), ws[1:].contiguous())
    torch.cuda.synchronize()
    assert not h[:-100].any() and torch.equal(h[-100:], want)
