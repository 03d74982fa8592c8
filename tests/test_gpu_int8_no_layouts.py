"""The int8 products, rows to int8 and the weighted dispatch with offsets and packed rows that are no layout's, every tensor
between guards: what is read and what is written is the tensors' own. Inside the tensors every value is the same, so that
every result is known whatever row it is taken from; in the guards and in the gaps between rows are values that would show."""
import numpy as np
import pytest
import torch

from paper_2607_06202_amd import epl
from tests.gpu_util import device
from tests.products_util import Packed

pytestmark = pytest.mark.gpu

NAN = float("nan")
BIG = 2 ** 31 - 1
AROUND = 128  # elements (1-D) or rows on either side


def between(shape, value, guard, dtype, pitch=0):
    """A tensor of `value`, rows `pitch` elements apart, inside a block of `guard` -> (tensor, block, mask of the tensor)."""
    rows = shape[0]
    block = torch.full((rows + 2 * AROUND, *shape[1:-1], pitch or shape[-1]) if len(shape) > 1 else (rows + 2 * AROUND,), guard,
                       dtype=dtype, device=device())
    mask = torch.zeros(block.shape, dtype=torch.bool, device=device())
    cut = (slice(AROUND, AROUND + rows),) + ((Ellipsis, slice(0, shape[-1])) if len(shape) > 1 else ())
    block[cut] = value
    mask[cut] = True
    return block[cut], block, mask


def assert_own(t, values, what):
    """Inside only the values, outside only the guard of 77."""
    view, block, mask = t
    assert bool((block[~mask] == 77).all()), what + ": written outside"
    assert bool(torch.stack([view == v for v in values]).any(0).all()), what + ": %s" % torch.unique(view)[:8].tolist()


@pytest.mark.parametrize("T", [16, 200, 600, 2400])  # a handful of rows; 64, 128 and 256 rows a tile
def test_offsets(T):
    E, K, N = 8, 80, 72
    pk = Packed(np.zeros((T, 1), np.int32), E, K, device(), row_pitch=128)
    bf = torch.bfloat16
    x, xs = between((T, K), 1, 127, torch.int8, 128)[0], between((T,), 1.0, NAN, torch.float32)[0]
    w, ws = between((E, N, K), 1, 127, torch.int8)[0], between((E, N), 1.0, NAN, torch.float32)[0]
    bias, res = between((E, N), 1.0, NAN, bf)[0], between((T, N), 2.0, NAN, bf, N + 8)[0]
    a = between((T, K), -3.0, NAN, bf, K + 8)[0]
    for off in ([0, -5, T + 100, 3, BIG, -BIG - 1, T, 1, BIG], [T] * 9, [-1] * 9, [5, 4, 3, 2, 1, 0, -1, -2, -3],
                [0, T, 0, T, 0, T, 0, T, 0], [T - 1] + [T] * 8, [0, 1] + [BIG] * 7, list(range(T - 9, T)), [0] * 8 + [T]):
        pk.L.expert_off.copy_(torch.tensor(off, dtype=torch.int32))
        out, h = between((T, N), 77, 77, bf, N + 16), between((T, N), 77, 77, bf)
        q, s = between((T, K), 77, 77, torch.int8, K + 16), between((T,), 77, 77, torch.float32)
        epl.experts_linear_int8(pk.cfg, x, xs, pk.L, w, ws, bias, res, out=out[0])
        epl.experts_gated_int8(pk.cfg, x, xs, pk.L, w, ws, w, ws, activation="none", h=h[0])
        epl.quantize_rows(pk.cfg, a, pk.L, q=q[0], q_scale=s[0])
        torch.cuda.synchronize()
        assert_own(out, (77, K + 3), "linear, %s" % off)
        assert_own(h, (77, K * K), "gated, %s" % off)
        assert_own(q, (77, -127), "rows, %s" % off)
        assert_own(s, (77, float(torch.tensor(3.0) / 127)), "scales, %s" % off)


@pytest.mark.parametrize("T,k,H", [(1, 2, 16), (37, 4, 272), (300, 8, 2064), (40, 32, 4112)])
def test_packed_rows(T, k, H):
    pitch, rows = -(-H // 64) * 64 + 64, T * k
    rng = np.random.default_rng(T)
    pk = Packed(rng.integers(0, 4, (T, k)).astype(np.int32), 4, H, device(), row_pitch=pitch)
    row = rng.integers(-3, rows + 3, (T, k))
    row[0, :2] = BIG, -BIG - 1
    row[-1, -1] = rows
    pk.L.pair_row.copy_(torch.from_numpy(row.astype(np.int32)))
    bf = torch.bfloat16
    x, w = between((T, H), 2.0, NAN, bf)[0], between((T, k), 1.5, NAN, torch.float32)[0]
    d = between((rows, H), 0.5, NAN, bf, pitch)[0]
    recv, q, s = between((rows, H), 77, 77, bf, pitch), between((rows, H), 77, 77, torch.int8, pitch), between((rows,), 77, 77, torch.float32)
    dx, dw = between((T, H), 77, 77, bf), between((T, k), 77, 77, torch.float32)
    epl.dispatch_weighted(pk.cfg, x, w, pk.L, recv=recv[0])
    epl.dispatch_int8(pk.cfg, x, pk.L, w, recv=q[0], recv_scale=s[0])
    epl.dispatch_backward(pk.cfg, d, x, w, pk.L, dx=dx[0], dtopk_w=dw[0])
    torch.cuda.synchronize()
    inside = torch.from_numpy((row >= 0) & (row < rows))
    hit = torch.zeros(rows, dtype=torch.bool)
    hit[torch.from_numpy(row)[inside]] = True
    for t, value in ((recv, 3.0), (q, 127), (s, float(torch.tensor(2.0) / 127 * 1.5))):
        assert_own(t, (77, value), "dispatch")
        got = (t[0] == value).cpu()
        assert torch.equal(got if got.dim() == 1 else got.all(1), hit)
    assert_own(dw, (0.0, float(H)), "dtopk_w")  # <2, 0.5> of H columns
    assert torch.equal(dw[0].cpu() == H, inside)
    assert bool((dx[1][~dx[2]] == 77).all())
    assert torch.equal(dx[0].cpu(), (0.75 * inside.sum(1)).bfloat16()[:, None].expand(T, H))
