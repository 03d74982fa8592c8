"""The int8 products on every tile shape with several tiles a workgroup, whose loads run on from one tile into the next: over
more than one group of 64 experts, ragged experts and experts without rows, short and long reductions. Whatever the
offsets hold, no access leaves the buffers. Activations at every bf16 value, relative to the result. Refused tensors."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import FEW, SLOPE, Packed, act, assert_within, rounded, routing_of_counts
from tests.test_gpu_activations import FLOOR, LIMIT, assert_close, exact, points, rows_of

pytestmark = pytest.mark.gpu

ONE = 2.0 ** -24

# (experts, rows each about, K, N): 64, 128 and 256 rows a tile by the rows each.
SHAPES = [(200, 20, 16, 1032), (200, 30, 272, 1544), (130, 45, 1040, 520), (70, 100, 144, 1288), (66, 135, 528, 776),
          (66, 200, 528, 776),
          (66, 300, 144, 1032), (20, 900, 656, 1544), (5, 5000, 16, 2056), (3, 6000, 2064, 776)]


def inputs(E, each, K, g, rng):
    counts = rng.integers(0, 2 * each, E)
    counts[rng.integers(0, E, max(E // 8, 1))] = 0
    counts[0], counts[-1] = each, 2 * each
    counts = [int(c) for c in counts]
    while sum(counts) < each * E:  # the kernels go by all rows there can be over all experts
        counts[int(rng.integers(0, E))] += each // 2
    pk = Packed(routing_of_counts(counts, E, 1, rng), E, 64, device())
    x = torch.randint(-127, 128, (pk.rows, K), generator=g, dtype=torch.int8).to(pk.dev)
    xs = (torch.rand(pk.rows, generator=g) * 0.02 + 0.001).to(pk.dev)
    return pk, x, xs


def weights(E, N, K, g, dev):
    return (torch.randint(-127, 128, (E, N, K), generator=g, dtype=torch.int8).to(dev),
            (torch.rand(E, N, generator=g) * 0.02 * K ** -0.5 + 1e-5).to(dev))


def product(pk, x, xs, w, ws, e, a, b):
    """On the GPU in 64 bits, where sums of these sizes are exact."""
    v = torch.matmul(x[a:b].double(), w[e].double().t().contiguous()) * xs[a:b].double()[:, None] * ws[e].double()
    return v.cpu()


@pytest.mark.parametrize("E,each,K,N", SHAPES)
def test_linear(E, each, K, N):
    g, rng = torch.Generator().manual_seed(E), np.random.default_rng(E)
    pk, x, xs = inputs(E, each, K, g, rng)
    w, ws = weights(E, N, K, g, pk.dev)
    bias = torch.randn(E, N, generator=g).bfloat16().to(pk.dev)
    res = pk.buffer(g, N)
    out, plain = pk.out(N, N + 8), pk.out(N)
    epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, bias, res, "silu", out=out)
    epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, out=plain)
    again = epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws)
    torch.cuda.synchronize()
    pk.assert_untouched(out, "out")
    pk.assert_untouched(plain, "plain")
    assert torch.equal(again[: pk.P], plain[: pk.P])
    for e, a, b in pk.experts():
        if a == b:
            continue
        v = product(pk, x, xs, w, ws, e, a, b)
        dv = 4 * ONE * v.abs()
        assert_within(plain[a:b], v, rounded(v, dv), "plain, expert %d" % e)
        v = v + bias[e].cpu().double()
        dv = dv + ONE * (v.abs() + dv)
        r = act("silu", v)
        err = SLOPE * dv + FEW * r.abs()
        r = r + res[a:b].cpu().double()
        err = err + ONE * (r.abs() + err)
        assert_within(out[a:b], r, rounded(r, err), "expert %d" % e)


@pytest.mark.parametrize("E,each,K,N", SHAPES)
def test_gated(E, each, K, N):
    g, rng = torch.Generator().manual_seed(E + 1), np.random.default_rng(E + 1)
    pk, x, xs = inputs(E, each, K, g, rng)
    cfg = epl.config(1, E, 1, K, pk.rows)
    (wg, gs), (wu, us) = weights(E, N, K, g, pk.dev), weights(E, N, K, g, pk.dev)
    h = pk.out(N)
    epl.experts_gated_int8(cfg, x, xs, pk.L, wg, gs, wu, us, "gelu", h=h)
    torch.cuda.synchronize()
    pk.assert_untouched(h, "h")
    for e, a, b in pk.experts():
        if a == b:
            continue
        v, u = product(pk, x, xs, wg, gs, e, a, b), product(pk, x, xs, wu, us, e, a, b)
        dv, du = 4 * ONE * v.abs(), 4 * ONE * u.abs()
        r = act("gelu", v)
        err = SLOPE * dv * (u.abs() + du) + (r.abs() + FEW) * du + FEW * (r * u).abs()
        assert_within(h[a:b], r * u, rounded(r * u, err), "expert %d" % e)


@pytest.mark.parametrize("E,T", [(8, 16), (8, 200), (8, 600), (8, 2400)])
def test_offsets_that_are_no_layouts(E, T):
    """expert_off is read on the device: whatever it holds, the rows read and written are the buffer's own."""
    dev = device()
    g = torch.Generator().manual_seed(T)
    pk = Packed(np.zeros((T, 1), np.int32), E, 64, dev)
    x = torch.randint(-127, 128, (T, 64), generator=g, dtype=torch.int8).to(dev)
    xs = torch.ones(T, device=dev)
    w, ws = weights(E, 72, 64, g, dev)
    for off in ([0, -5, T + 100, 3, 2 ** 31 - 1, -2 ** 31, T, 1, 2 ** 31 - 1], [T] * 9, [-1] * 9, [5, 4, 3, 2, 1, 0, -1, -2, -3],
                [0, T, 0, T, 0, T, 0, T, 0]):
        pk.L.expert_off.copy_(torch.tensor(off, dtype=torch.int32))
        block = torch.full((T + 200, 72), 77.0, dtype=torch.bfloat16, device=dev)
        out = block[100 : 100 + T]
        epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, out=out)
        epl.experts_gated_int8(pk.cfg, x, xs, pk.L, w, ws, w, ws, h=out)
        q = torch.full((T + 200, 80), 77, dtype=torch.int8, device=dev)
        s = torch.full((T + 200,), 77.0, device=dev)
        epl.quantize_rows(pk.cfg, torch.randn(T, 80, device=dev).bfloat16(), pk.L, q=q[100 : 100 + T], q_scale=s[100 : 100 + T])
        torch.cuda.synchronize()
        for t in (block, q, s):
            assert bool((t[:100] == 77).all()) and bool((t[100 + T:] == 77).all()), off


@pytest.mark.parametrize("E", [16, 160, 64, 8])  # few rows; 64, 128 and 256 rows a tile
@pytest.mark.parametrize("name", ["silu", "gelu", "relu", "none"])
def test_activations(name, E):
    v = points(LIMIT[name]) if name in ("silu", "gelu") else points(100.0)
    if E == 16:
        v = torch.linspace(-LIMIT[name] * 0.9, LIMIT[name] * 0.1, 16).bfloat16() if name in ("silu", "gelu") else v[::500][:16]
    pk = rows_of(v, E)
    T, per = v.numel(), v.numel() // E
    assert (T <= 16) == (E == 16) and (E != 160 or per < 56) and (E != 64 or 56 <= per < 144) and (E != 8 or per >= 144)
    x = torch.zeros(T, 128, dtype=torch.int8, device=pk.dev)
    x[:, 0] = 1
    w = torch.zeros(E, 8, 128, dtype=torch.int8, device=pk.dev)
    w[:, :, 0] = 1
    s, ws = v.float().to(pk.dev), torch.ones(E, 8, device=pk.dev)
    out = epl.experts_linear_int8(pk.cfg, x, s, pk.L, w, ws, activation=name)
    h = epl.experts_gated_int8(pk.cfg, x, s, pk.L, w, ws, w, ws, activation=name)
    torch.cuda.synchronize()
    want, _, err = exact(name, v)
    assert bool((out == out[:, :1]).all()) and bool((h == h[:, :1]).all())
    assert_close(out[:, 0], want, err, name, v)
    up = v.double()  # the up projection of the same rows
    assert_close(h[:, 0], want * up, (err + FEW * want.abs()) * up.abs() + FLOOR * up.abs(), "gated " + name, v)


def test_infinite_arguments():
    """A scale can pass what a product's value may be: infinities go through the activations as in 64 bits."""
    for T in (4, 40, 600, 2400):
        pk = Packed(np.zeros((T, 1), np.int32), 1, 64, device())
        x = torch.ones(T, 64, dtype=torch.int8, device=pk.dev)
        w, ws = torch.ones(1, 8, 64, dtype=torch.int8, device=pk.dev), torch.full((1, 8), 1e30, device=pk.dev)
        s = torch.full((T,), 1e30, device=pk.dev)
        for name in ("silu", "gelu", "relu", "none"):
            out = epl.experts_linear_int8(pk.cfg, x, s, pk.L, w, ws, activation=name)
            low = epl.experts_linear_int8(pk.cfg, x, -s, pk.L, w, ws, activation="relu")
            torch.cuda.synchronize()
            assert bool((out == float("inf")).all()), (T, name)
            assert not low.any()


def test_refused_tensors():
    """What the binding refuses before the call: types, shapes, strides, devices and layouts that do not fit."""
    dev = device()
    pk = Packed(np.zeros((8, 2), np.int32), 4, 64, dev, row_pitch=128)
    cfg, L = pk.cfg, pk.L
    x, tw = torch.zeros(8, 64, dtype=torch.bfloat16, device=dev), torch.ones(8, 2, device=dev)
    d = torch.zeros(16, 128, dtype=torch.bfloat16, device=dev)[:, :64]
    q, s = torch.zeros(16, 128, dtype=torch.int8, device=dev)[:, :64], torch.zeros(16, device=dev)
    w, ws = torch.zeros(4, 32, 64, dtype=torch.int8, device=dev), torch.zeros(4, 32, device=dev)
    out = torch.zeros(16, 32, dtype=torch.bfloat16, device=dev)
    other = Packed(np.zeros((9, 2), np.int32), 4, 64, dev).L
    calls = {
        "weighted": (lambda **k: epl.dispatch_weighted(cfg, k["x"], k["tw"], k["L"], recv=k["d"]), "x tw L d"),
        "backward": (lambda **k: epl.dispatch_backward(cfg, k["d"], k["x"], k["tw"], k["L"], dx=k["dx"], dtopk_w=k["dw"]),
                     "x tw L d dx dw"),
        "int8": (lambda **k: epl.dispatch_int8(cfg, k["x"], k["L"], k["tw"], recv=k["q"], recv_scale=k["s"]), "x tw L q s"),
        "quantize": (lambda **k: epl.quantize_rows(cfg, k["d"], k["L"], q=k["q"], q_scale=k["s"]), "d L q s"),
        "gated": (lambda **k: epl.experts_gated_int8(cfg, k["q"], k["s"], k["L"], k["w"], k["ws"], k["w"], k["ws"],
                                                     h=k["out"]), "q s L w ws out"),
        "linear": (lambda **k: epl.experts_linear_int8(cfg, k["q"], k["s"], k["L"], k["w"], k["ws"], residual=k["out"],
                                                       out=k["y"]), "q s L w ws out y"),
    }
    good = dict(x=x, tw=tw, L=L, d=d, q=q, s=s, w=w, ws=ws, out=out, dx=torch.zeros_like(x), dw=torch.zeros_like(tw),
                y=torch.zeros_like(out))
    for name, (call, used) in calls.items():
        call(**good)
        for n in used.split():
            if n == "L":
                with pytest.raises(ValueError):
                    call(**dict(good, L=other))
                continue
            t = good[n]
            bad = [t.float() if t.dtype != torch.float32 else t.bfloat16(), t.cpu(), t[:-1], t[..., :-8] if t.dim() > 1 else t[:4],
                   t.unsqueeze(0)]
            if t.dim() > 1:
                bad.append(torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=dev)[..., ::2])
                bad.append(torch.zeros(1, *t.shape[1:], dtype=t.dtype, device=dev).expand(t.shape))
            for b in bad:
                with pytest.raises(ValueError):
                    call(**dict(good, **{n: b}))
        torch.cuda.synchronize()
    with pytest.raises(ValueError):
        epl.quantize_weights(torch.zeros(4, 32, 64, dtype=torch.bfloat16, device=dev)[:, :, ::2])
    with pytest.raises(epl.EplError, match="UNSUPPORTED"):
        epl.quantize_weights(torch.zeros(4, 32, 24, dtype=torch.bfloat16, device=dev))
    with pytest.raises(epl.EplError, match="INVALID"):
        epl.dispatch_backward(cfg, d, x, tw, L, dx=torch.zeros_like(x), dtopk_w=tw)
    with pytest.raises(ValueError):
        epl.experts_gated_int8(cfg, q, s, L, w, ws, w[:, :16], ws)
