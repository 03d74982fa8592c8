"""The router (epl_route, epl_route_backward) against 64-bit references: choices equal, weights and gradients within
their bounds; ties, masks, NaN and infinite logits, near-ties of biased scores, more choices than experts are left."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}


def reference(l, bias, k, score, normalize, scale):
    """Choices and weights in 64 bits, one token at a time."""
    l = l.double().numpy()
    T, E = l.shape
    idx = np.full((T, k), -1, np.int32)
    w = np.zeros((T, k))
    p = np.zeros((T, E))
    for t in range(T):
        ok = l[t] > -np.inf  # false for NaN
        if ok.any():
            if score == "sigmoid":
                with np.errstate(over="ignore"):
                    p[t, ok] = 1 / (1 + np.exp(-l[t, ok]))
            else:
                m = l[t, ok].max()
                with np.errstate(invalid="ignore"):
                    ex = np.where(l[t, ok] == m, 1.0, np.exp(l[t, ok] - m))
                p[t, ok] = ex / ex.sum()
        key = l[t] if bias is None else p[t] + bias.double().numpy()
        cand = [e for e in range(E) if ok[e] and key[e] > -np.inf]
        pick = sorted(cand, key=lambda e: (-key[e], e))[:k]
        idx[t, : len(pick)] = pick
        w[t, : len(pick)] = p[t, pick]
        if normalize:
            s = w[t].sum()
            w[t] = w[t] / s if s > 0 else 0.0
    return idx, w * scale, p


def check(l, k, bias=None, score="softmax", normalize=True, scale=1.0):
    dev = device()
    T, E = l.shape
    cfg = epl.config(1, E, k, 8, T)
    idx, w = epl.route(cfg, l.to(dev), None if bias is None else bias.to(dev), score, normalize, scale)
    torch.cuda.synchronize()
    want_i, want_w, _ = reference(l, bias, k, score, normalize, scale)
    np.testing.assert_array_equal(idx.cpu().numpy(), want_i)
    # exp 1 ulp and its argument, a sum of E <= 1024 terms (22 additions deep), two divisions, the scale: 32 roundings
    np.testing.assert_allclose(w.cpu().numpy(), want_w, rtol=32 * 2.0 ** -24, atol=1e-37)
    return idx, w


@pytest.mark.parametrize("E", [1, 5, 64, 65, 128, 160, 256, 500, 1024])
@pytest.mark.parametrize("score,normalize,biased", [("softmax", True, False), ("softmax", False, True),
                                                     ("sigmoid", True, True), ("sigmoid", False, False),
                                                     ("softmax", True, True)])
def test_choices_and_weights(E, score, normalize, biased):
    g = torch.Generator().manual_seed(E)
    for dt in (torch.float32, torch.bfloat16):
        l = (torch.randn(67, E, generator=g) * 2).to(dt)
        bias = torch.randn(E, generator=g) * 0.1 if biased else None
        for k in (1, 8, 32):
            check(l, k, bias, score, normalize, 2.5)


def test_masks_ties_and_special_values():
    g = torch.Generator().manual_seed(1)
    inf, nan = float("inf"), float("nan")
    l = torch.randn(16, 130, generator=g)
    l[0] = -inf                      # nothing left
    l[1, 3:] = -inf                  # fewer experts than choices
    l[2] = 0.5                       # all equal: the lowest indices
    l[3, ::2] = 0.0
    l[3, 1::2] = -0.0                # zeros of both signs are equal
    l[4, 7] = nan                    # a NaN is masked
    l[5, [100, 9]] = inf             # two maxima
    l[6] = torch.finfo(torch.float32).min  # the lowest finite value is a logit like any other
    l[7, 5:] = torch.finfo(torch.float32).min
    l[8] = nan
    l[9] = -200.0                    # sigmoid underflows to nothing
    l[10, 1:] = -1000.0              # softmax underflows beside one expert
    bias = torch.randn(130, generator=g) * 0.1
    bias[11], bias[12], bias[13] = nan, -inf, inf
    for score in ("softmax", "sigmoid"):
        for normalize in (True, False):
            check(l, 6, None, score, normalize)
            check(l, 6, bias, score, normalize)


def test_near_ties_of_biased_scores_follow_64_bits():
    """Scores one fp32 rounding apart and below: the bias undoes the difference of the scores up to 1e-9."""
    g = torch.Generator().manual_seed(2)
    T, E = 64, 96
    l = torch.randn(1, E, generator=g).expand(T, E).contiguous()
    for score in ("sigmoid", "softmax"):
        p = torch.sigmoid(l[0].double()) if score == "sigmoid" else torch.softmax(l[0].double(), 0)
        bias = (0.5 - p).float()     # every key is 0.5 to within half a unit of the bias
        check(l, 8, bias, score, True)


def test_equal_logits_and_bias_tie_to_the_lowest_index():
    l = torch.zeros(5, 200)
    l[:, 50:60] = 1.0
    bias = torch.zeros(200)
    check(l, 12, bias, "sigmoid", True)
    check(l.bfloat16(), 12, bias, "softmax", False)


@pytest.mark.parametrize("E", [5, 64, 130, 256, 1024])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,normalize", [("softmax", True), ("softmax", False), ("sigmoid", True),
                                             ("sigmoid", False)])
def test_gradient(E, dt, score, normalize):
    """Against autograd in 64 bits. The bound counts 64 roundings of the largest term of the sums: dl is a product
    of scores with differences of dw, each of at most scale * max|dw| * k."""
    dev = device()
    g = torch.Generator().manual_seed(E + 7)
    T, k, scale = 33, min(E, 8), 2.5
    l = (torch.randn(T, E, generator=g) * 2).to(dt)
    l[0] = float("-inf")
    l[1, 1:] = float("-inf")
    cfg = epl.config(1, E, k, 8, T)
    idx, _ = epl.route(cfg, l.to(dev), None, score, normalize, scale)
    idx[2, 0] = -1
    idx[3, 0] = E + 5
    if k > 1:
        idx[4, 1] = idx[4, 0]       # the same expert twice
    dw = torch.randn(T, k, generator=g)
    got = epl.route_backward(cfg, l.to(dev), idx, dw.to(dev), score, normalize, scale)
    torch.cuda.synchronize()
    assert got.dtype == dt
    i = idx.cpu().long()
    valid = (i >= 0) & (i < E)
    valid &= l.double().gather(1, i.clamp(0, E - 1)) > float("-inf")
    z = l.double().clone()
    dead = torch.isneginf(z)
    z[dead] = -1e9                   # a finite stand-in whose score is 0
    z[0] = 0.0
    z.requires_grad_(True)
    p = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, 1)
    w = torch.where(valid, p.gather(1, i.clamp(0, E - 1)), 0.0)
    if normalize:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    (w * dw.double() * scale).sum().backward()
    want = z.grad.masked_fill(dead, 0.0)
    err = (got.cpu().double() - want).abs()
    bound = 64 * 2.0 ** -24 * scale * dw.abs().double().sum(1, keepdim=True) + HALF[dt] * want.abs() * 1.001 + 1e-37
    assert bool((err <= bound).all()), float((err - bound).max())
    assert not got[0].any()


def test_gradient_against_differences():
    dev = device()
    g = torch.Generator().manual_seed(9)
    T, E, k = 4, 12, 3
    l = torch.randn(T, E, generator=g)
    dw = torch.randn(T, k, generator=g)
    cfg = epl.config(1, E, k, 8, T)
    for score in ("softmax", "sigmoid"):
        for normalize in (True, False):
            idx, _ = epl.route(cfg, l.to(dev), None, score, normalize)
            got = epl.route_backward(cfg, l.to(dev), idx, dw.to(dev), score, normalize).cpu().double()

            def loss(z):
                p = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, 1)
                w = p.gather(1, idx.cpu().long())
                return ((w / w.sum(1, keepdim=True) if normalize else w) * dw.double()).sum()

            eps = 1e-5  # central difference in 64 bits: error eps^2 * |third derivative| < 1e-8
            for t, e in [(0, 0), (1, 5), (2, 11), (3, int(idx[3, 0])), (0, int(idx[0, 2]))]:
                d = torch.zeros(T, E, dtype=torch.float64)
                d[t, e] = eps
                diff = float(loss(l.double() + d) - loss(l.double() - d)) / (2 * eps)
                assert abs(diff - float(got[t, e])) < 1e-5, (score, normalize, t, e)


def test_no_tokens():
    dev = device()
    cfg = epl.config(1, 16, 2, 8, 0)
    idx, w = epl.route(cfg, torch.empty(0, 16, device=dev))
    assert idx.shape == (0, 2) and w.shape == (0, 2)
    assert epl.route_backward(cfg, torch.empty(0, 16, device=dev), idx, w).shape == (0, 16)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_one_renormalised_choice_has_no_gradient(score):
    """Its weight is p / p = 1 whatever the logits are, so the gradient is exactly zero."""
    dev = device()
    cfg = epl.config(1, 40, 1, 8, 33)
    l = torch.randn(33, 40, generator=torch.Generator().manual_seed(3)).to(dev)
    idx, w = epl.route(cfg, l, score=score)
    d = epl.route_backward(cfg, l, idx, torch.full((33, 1), 3.7, device=dev), score=score)
    torch.cuda.synchronize()
    assert bool((w == 1).all()) and not d.any()
