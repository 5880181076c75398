"""Layer norm's gradient of more rows than the GPU holds at once, so that groups
of lanes and blocks walk over rows and end partway through a step: the sums over
rows exactly, every row's gradient against the formula in 64 bits."""
import pytest
import torch

from paper_2207_10731_amd import pss
from rows_common import HALF, U, chain, make_drop

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# groups of 1, 2, 4, 8, 16, 32 and 64 lanes (one span and two), blocks of one span
# and two, the wide form; two rounds of rows, three and more
SHAPES = [(600007, 8), (300001, 16), (400003, 5), (70001, 30), (140003, 32), (40001, 33), (100003, 33),
          (53251, 128), (20011, 250), (12007, 500), (5003, 520), (5003, 1000), (3001, 1500), (1503, 2051),
          (1100, 4096), (1030, 5000), (790, 8192), (777, 9001), (600, 12288), (4100, 16390)]


def _whole(shape, low, high, dtype, g):
    return torch.randint(low, high, shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rows_walked_over(rows, cols, dtype):
    """grad_out 1 to 3 and s -2 to 2 with mean 0 and rstd 1: z = s, and every
    partial sum over rows is a whole number below 2^24, exact in any order."""
    assert rows * 6 < 2**24
    g = torch.Generator("cuda").manual_seed(cols)
    dy, s = _whole((rows, cols), 1, 4, dtype, g), _whole((rows, cols), -2, 3, dtype, g)
    up = _whole((rows, cols), -1, 2, dtype, g)
    w = torch.rand(cols, generator=g, device="cuda") + 0.5
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    drop = make_drop(0.25)
    gx, gr = torch.full_like(dy, 77.0), torch.full_like(dy, 77.0)
    gw, gb = (torch.full((cols,), 77.0, device="cuda") for _ in range(2))
    pss.pss_layer_norm_backward(dy, s, w, mean, rstd, gx, gw, gb, grad_sum=up, dropout=drop,
                                grad_residual=gr)
    assert torch.equal(gb, dy.double().sum(0).float())
    assert torch.equal(gw, (dy.double() * s.double()).sum(0).float())
    ones, kept = torch.ones_like(dy), torch.empty_like(dy)
    pss.pss_dropout(ones, drop, kept)
    n = max(1, (1 << 22) // cols)
    for r in range(0, rows, n):
        at = slice(r, min(r + n, rows))
        z, h = s[at].double(), dy[at].double() * w.double()
        hz = h * z
        plain = h - h.mean(1, keepdim=True) - z * hz.mean(1, keepdim=True)
        ref = plain + up[at].double()
        # the two sums are off by chain u times their magnitudes, and ten more
        # roundings of the formula's terms
        err = (chain(cols) + 10) * U * (h + h.mean(1, keepdim=True)
                                        + z.abs() * hz.abs().mean(1, keepdim=True))
        err = err + U * (ref.abs() + up[at].double().abs())
        for got, v, e, what in (
                (gr, ref, err, "grad_residual"),
                (gx, torch.where(kept[at] == 0, 0.0, ref / 0.75),
                 torch.where(kept[at] == 0, 0.0, err / 0.75 + 2 * U * ref.abs() / 0.75), "grad_x")):
            tol = e + HALF[dtype] * (v.abs() + e) + 1e-38
            bad = ~((got[at].double() - v).abs() <= tol)
            assert not bool(bad.any()), (what, r, bad.nonzero()[:3].tolist())
    again = [torch.empty_like(gw), torch.empty_like(gb)]
    pss.pss_layer_norm_backward(dy, s, w, mean, rstd, gx, *again)
    assert torch.equal(again[0], gw) and torch.equal(again[1], gb)
