"""epl_dispatch_weighted bit for bit and its gradient against 64 bits: invalid pairs, padded tokens, pitches, many choices, in
place; a layer that weights the experts' inputs, forward and backward, against autograd and differences, on another
stream and in a captured graph."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import BF16_HALF_STEP, Packed, assert_within, sum_error, weights

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8, 1, 1, 8, 0), (2, 8, 2, 9, 264, 320), (4, 16, 8, 33, 1024, 0), (4, 64, 8, 16, 7168, 7936),
          (1, 40, 12, 21, 2056, 0), (2, 64, 32, 5, 520, 576), (8, 32, 4, 300, 72, 0), (1, 8, 2, 3, 70000, 0),
          (1, 16, 4, 9, 5120, 0), (1, 16, 3, 5, 8192, 8256), (1, 16, 6, 7, 4104, 0), (1, 16, 1, 40, 7168, 0)]


def inputs(R, E, k, Tr, H, pitch):
    dev = device()
    g = torch.Generator().manual_seed(H + k)
    idx = np.random.default_rng(k).integers(-1, E + 1, (R * Tr, k)).astype(np.int32)  # some invalid, some twice
    if Tr > 2:
        idx[-2:] = -1
    pk = Packed(idx, E, H, dev, R=R, row_pitch=pitch)
    x = torch.randn(R * Tr, H, generator=g).bfloat16()
    w = torch.randn(R * Tr, k, generator=g)
    row = pk.L.pair_row.cpu().long()
    w[row < 0] = float("nan")  # not looked at
    return pk, g, x, w, row


@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape):
    pk, _, x, w, row = inputs(*shape)
    recv = pk.out(shape[4], shape[5])
    epl.dispatch_weighted(pk.cfg, x.to(pk.dev), w.to(pk.dev), pk.L, recv=recv)
    new = epl.dispatch_weighted(pk.cfg, x.to(pk.dev), w.to(pk.dev), pk.L)
    torch.cuda.synchronize()
    tok, j = (row >= 0).nonzero(as_tuple=True)
    assert torch.equal(recv.cpu()[row[tok, j]], (w[tok, j][:, None] * x[tok].float()).bfloat16())
    assert torch.equal(new[: pk.P], recv[: pk.P])
    pk.assert_untouched(recv, "recv")


def test_weights_of_one_are_dispatch_and_infinities_stay():
    pk, _, x, w, row = inputs(2, 8, 2, 9, 264, 320)
    x[1, 3], x[2, 4] = float("inf"), float("nan")
    plain, _ = epl.dispatch(pk.cfg, x.to(pk.dev), pk.L)
    ones = epl.dispatch_weighted(pk.cfg, x.to(pk.dev), torch.ones_like(w).to(pk.dev), pk.L)
    zeros = epl.dispatch_weighted(pk.cfg, x.to(pk.dev), torch.zeros_like(w).to(pk.dev), pk.L)
    torch.cuda.synchronize()
    bits = lambda t: torch.nan_to_num(t[: pk.P].float(), 12345.0, 1e38, -1e38)
    assert torch.equal(bits(plain), bits(ones))
    assert not torch.nan_to_num(zeros[: pk.P].float()).any()


@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape):
    R, E, k, Tr, H, pitch = shape
    pk, g, x, w, row = inputs(*shape)
    d = pk.buffer(g, H, pitch)  # NaN behind the last row and in the gaps
    xd, wd = x.to(pk.dev), w.to(pk.dev)
    dx, dw = epl.dispatch_backward(pk.cfg, d, xd, wd, pk.L)
    same = xd.clone()
    _, dw2 = epl.dispatch_backward(pk.cfg, d, same, wd, pk.L, dx=same)  # in place
    combined = epl.combine(pk.cfg, d, wd, pk.L)
    torch.cuda.synchronize()
    assert torch.equal(dw, dw2) and torch.equal(same, dx)
    assert torch.equal(dx, combined)
    assert not dw.cpu()[row < 0].any()
    tok, j = (row >= 0).nonzero(as_tuple=True)
    a, b = x.double()[tok], d.cpu().double()[row[tok, j]]
    assert_within(dw.cpu()[tok, j], (a * b).sum(1), sum_error(H + 2, (a * b).abs().sum(1)) + 1e-37, "dtopk_w")


def test_no_tokens():
    dev = device()
    cfg = epl.config(1, 4, 3, 64, 0)
    L = epl.alloc_layout(cfg, dev)
    x, w = torch.zeros(1, 64, dtype=torch.bfloat16, device=dev), torch.zeros(1, 3, device=dev)
    epl.dispatch_weighted(cfg, x, w, L)
    epl.dispatch_backward(cfg, x, x, w, L)
    torch.cuda.synchronize()


class Layer:
    """Experts that take weighted inputs: y = sum_j E_j(w_j x), with gated experts; forward and backward."""

    def __init__(self, R=2, E=16, k=4, Tr=40, H=128, I=192, pitch=192, seed=0, pad=3):
        g = torch.Generator().manual_seed(seed)
        self.cfg = epl.config(R, E, k, H, Tr, "bf16", pitch)
        T = R * Tr
        logits = torch.randn(T, E, generator=g)
        logits.view(R, Tr, E)[:, Tr - pad:] = float("-inf")
        self.host = dict(logits=logits, x=torch.randn(T, H, generator=g).bfloat16(), wg=weights(g, E, I, H, "cpu"),
                         wu=weights(g, E, I, H, "cpu"), wd=weights(g, E, H, I, "cpu"),
                         dout=torch.randn(T, H, generator=g).bfloat16())
        self.d = {n: t.to(device()) for n, t in self.host.items()}

    def forward(self):
        cfg, d = self.cfg, self.d
        idx, w = epl.route(cfg, d["logits"], score="sigmoid")
        L = epl.layout(cfg, idx)
        recv = epl.dispatch_weighted(cfg, d["x"], w, L)
        h, pre = epl.experts_gated(cfg, recv, L, d["wg"], d["wu"], keep_pre=True)
        y, _ = epl.experts_linear(cfg, h, L, d["wd"])
        return epl.combine(cfg, y, torch.ones_like(w), L), (idx, w, L, recv, h, pre, y)

    def backward(self, kept):
        cfg, d = self.cfg, self.d
        idx, w, L, recv, h, pre, y = kept
        dy, _ = epl.combine_backward(cfg, d["dout"], y, torch.ones_like(w), L)
        dh, dwd, _ = epl.experts_linear_backward(cfg, dy, h, L, d["wd"])
        drecv, dwg, dwu = epl.experts_gated_backward(cfg, dh, pre, recv, L, d["wg"], d["wu"])
        dx, dw = epl.dispatch_backward(cfg, drecv, d["x"], w, L)
        return dict(x=dx, logits=epl.route_backward(cfg, d["logits"], idx, dw, score="sigmoid"), wg=dwg, wu=dwu, wd=dwd)

    def value(self, v, idx):
        """The output in 64 bits from the values v, for these choices."""
        dead = torch.isneginf(self.host["logits"]).all(1)[:, None]
        p = torch.sigmoid(torch.where(dead, 0.0, v["logits"])).gather(1, idx.clamp_min(0)) * (idx >= 0)
        w = p / p.sum(1, keepdim=True).clamp_min(1e-300)
        out = torch.zeros_like(v["x"])
        for j in range(idx.shape[1]):
            for e in range(self.cfg.num_experts):
                t = (idx[:, j] == e).nonzero()[:, 0]
                if t.numel():
                    xe = w[t, j][:, None] * v["x"][t]
                    h = torch.nn.functional.silu(xe @ v["wg"][e].T) * (xe @ v["wu"][e].T)
                    out = out.index_add(0, t, h @ v["wd"][e].T)
        return out

    def values(self):
        v = {n: t.double() for n, t in self.host.items() if n != "dout"}
        v["logits"] = torch.nan_to_num(v["logits"], neginf=0.0)
        return v


def relative(got, want):
    return float((got.cpu().double() - want).norm() / want.norm().clamp_min(1e-30))


# As in the layer with weights behind the experts: bf16 roundings on the way, each of relative size at most 2^-8; here recv is
# one of them (forward recv, h, y, out; backward dy is exact, dh, dpre, drecv, dx, and what the forward pass kept), at most
# nine for any gradient, with silu's slope of 1.1 for those that pass through the gate; recv's goes into the gate and the up
# projection, so it counts twice.
WAY = 10 * BF16_HALF_STEP * 1.1


@pytest.mark.parametrize("shape", [dict(), dict(R=1, E=8, k=2, Tr=1, H=64, I=64, pitch=0, pad=0),
                                   dict(R=4, E=32, k=8, Tr=130, H=264, I=136, pitch=320, pad=7, seed=3),
                                   dict(R=2, E=8, k=3, Tr=17, H=128, I=128, pitch=0, pad=17, seed=4)],
                         ids=["small", "one_token", "odd", "all_padding"])
def test_layer_forward_and_backward(shape):
    layer = Layer(**shape)
    out, kept = layer.forward()
    grads = layer.backward(kept)
    torch.cuda.synchronize()
    v = layer.values()
    for t in v.values():
        t.requires_grad_(True)
    want = layer.value(v, kept[0].cpu().long())
    if not want.requires_grad:  # nothing but padding
        assert not out.any() and all(not g.any() for g in grads.values())
        return
    want.backward(layer.host["dout"].double())
    assert relative(out, want.detach()) <= WAY
    for n, g in grads.items():
        assert torch.isfinite(g).all(), n
        assert relative(g, v[n].grad) <= WAY, (n, relative(g, v[n].grad))


def test_gradients_against_differences():
    """Directional derivatives of the 64-bit layer against the kernels' gradients; the central difference's own error is of
    the order of eps^2."""
    layer = Layer(R=1, E=4, k=2, Tr=12, H=64, I=64, pitch=0, pad=0, seed=5)
    _, kept = layer.forward()
    grads = layer.backward(kept)
    torch.cuda.synchronize()
    idx, base = kept[0].cpu().long(), layer.values()
    loss = lambda v: float((layer.value(v, idx) * layer.host["dout"].double()).sum())
    g = torch.Generator().manual_seed(6)
    for n, grad in grads.items():
        step = torch.randn(base[n].shape, generator=g, dtype=torch.float64)
        eps = 1e-5
        diff = (loss({**base, n: base[n] + eps * step}) - loss({**base, n: base[n] - eps * step})) / (2 * eps)
        got = float((grad.cpu().double() * step).sum())
        assert abs(diff - got) <= WAY * float(grad.cpu().double().norm() * step.norm()) + 1e-6, (n, diff, got)


def test_another_stream_and_a_captured_graph():
    layer = Layer(seed=8)
    torch.cuda.synchronize()
    out, kept = layer.forward()
    grads = layer.backward(kept)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out2, kept2 = layer.forward()
        grads2 = layer.backward(kept2)
    s.synchronize()
    assert torch.equal(out, out2) and all(torch.equal(grads[n], grads2[n]) for n in grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, kept = layer.forward()
        grads = layer.backward(kept)
    for seed in range(4):
        other = Layer(seed=20 + seed, pad=seed)
        for n, t in layer.d.items():
            t.copy_(other.d[n])
        graph.replay()
        torch.cuda.synchronize()
        want, kept2 = other.forward()
        want_grads = other.backward(kept2)
        torch.cuda.synchronize()
        assert torch.equal(out, want), seed
        for n in grads:
            assert torch.equal(grads[n], want_grads[n]), (seed, n)


def test_offsets_past_32_bits():
    """Packed rows past 4 GiB, forward and backward: the last ones against the same alone."""
    dev = device()
    g = torch.Generator().manual_seed(9)
    rows, pitch = 70000, 32768  # 4.6 GB
    idx = np.zeros((rows, 1), np.int32)
    idx[-100:] = 1
    far = Packed(idx, 2, 64, dev, row_pitch=pitch)
    x = torch.zeros(rows, 64, dtype=torch.bfloat16, device=dev)
    x[-100:] = torch.randn(100, 64, generator=g).bfloat16().to(dev)
    w = torch.full((rows, 1), 0.37, device=dev)
    recv = torch.empty(rows, pitch, dtype=torch.bfloat16, device=dev)[:, :64]
    epl.dispatch_weighted(far.cfg, x, w, far.L, recv=recv)
    torch.cuda.synchronize()
    assert not recv[:-100].any() and torch.equal(recv[-100:], (w[-100:] * x[-100:].float()).bfloat16())
    dx, dw = epl.dispatch_backward(far.cfg, recv, x, w, far.L)
    near = Packed(np.zeros((100, 1), np.int32), 1, 64, dev)
    want = epl.dispatch_backward(near.cfg, recv[-100:].contiguous(), x[-100:].contiguous(), w[-100:].contiguous(), near.L)
    torch.cuda.synchronize()
    assert not dx[:-100].any() and not dw[:-100].any()
    assert torch.equal(dx[-100:], want[0]) and torch.equal(dw[-100:], want[1])
