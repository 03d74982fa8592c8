"""epl_combine_backward against a 64-bit reference: invalid pairs, padded tokens, pitches, many choices, in place."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import Packed, assert_within, rounded, sum_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,E,k,Tr,H,pitch", [(1, 8, 1, 1, 8, 0), (2, 8, 2, 9, 264, 320), (4, 16, 8, 33, 1024, 0),
                                              (4, 64, 8, 16, 7168, 7936), (1, 40, 12, 21, 2056, 0),
                                              (2, 64, 32, 5, 520, 576), (1, 4, 3, 0, 64, 0)])
def test_against_reference(R, E, k, Tr, H, pitch):
    dev = device()
    g = torch.Generator().manual_seed(H + k)
    rng = np.random.default_rng(k)
    idx = rng.integers(-1, E + 1, (R * Tr, k)).astype(np.int32)  # some invalid, some twice
    if Tr > 2:
        idx[-2:] = -1
    pk = Packed(idx, E, H, dev, R=R, row_pitch=pitch) if Tr else None
    cfg = pk.cfg if pk else epl.config(R, E, k, H, 0)
    L = pk.L if pk else epl.alloc_layout(cfg, dev)
    T = R * Tr
    dout = torch.randn(max(T, 1), H, generator=g).bfloat16().to(dev)
    w = torch.randn(max(T, 1), k, generator=g).to(dev)
    if not pk:
        y = torch.zeros(1, H, dtype=torch.bfloat16, device=dev)
        epl.combine_backward(cfg, dout, y, w, L)
        torch.cuda.synchronize()
        return
    y = pk.buffer(g, H, pitch)
    dy = pk.out(H, pitch)
    _, dw = epl.combine_backward(cfg, dout, y, w, L, dy=dy)
    same = y.as_strided((pk.rows, pitch or H), (pitch or H, 1)).clone()[:, :H]
    _, dw2 = epl.combine_backward(cfg, dout, same, w, L, dy=same)  # in place
    torch.cuda.synchronize()
    assert torch.equal(dw, dw2) and torch.equal(same[: pk.P], dy[: pk.P])
    pk.assert_untouched(dy, "dy")
    row = L.pair_row.cpu().long()
    assert not dw.cpu()[row < 0].any()
    tok, j = (row >= 0).nonzero(as_tuple=True)
    r = row[tok, j]
    d, yd = dout.cpu().double()[tok], y.cpu().double()[r]
    want = w.cpu().double()[tok, j][:, None] * d
    assert_within(dy[r.to(dev)], want, rounded(want, 2.0 ** -23 * want.abs()), "dy")
    want = (d * yd).sum(1)
    assert_within(dw.cpu()[tok, j], want, sum_error(H + 2, (d * yd).abs().sum(1)) + 1e-37, "dtopk_w")
