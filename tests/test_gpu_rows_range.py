"""Layer norm of rows whose values lie far out in float32's range: finite rows
give finite results at every width, the group, block and wide forms alike."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss
from rows_common import EPS, U, make_rows, norm_grad_ref, numpy64, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
BIG = 2.0**65  # its square is beyond float32, the sum of a row of them is not


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1000, 1024, 1032, 2048, 2051, 4096, 5000, 8192, 9001, 16384, 20000,
                                  32768])
def test_forward_of_large_values(cols, dtype):
    x = torch.randn(5, cols, device="cuda").to(dtype)
    x[0], x[1], x[2], x[3] = BIG, -BIG, 0.0, 0.0
    x[2, cols // 2] = 1e30
    x[3, cols - 1] = -1e30
    w, b = torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
    out = torch.empty_like(x)
    mean, rstd = (torch.empty(5, device="cuda") for _ in range(2))
    pss.pss_layer_norm_forward(x, w, b, EPS, out, mean, rstd)
    assert bool(out.isfinite().all()) and bool(mean.isfinite().all()) and bool(rstd.isfinite().all())
    for r in (2, 3):  # squares beyond float32: rstd = 0, and every difference is finite
        assert rstd[r] == 0 and torch.equal(out[r], b.to(dtype))
    if cols & (cols - 1) == 0:  # sums of n 2^65, n < 2^24, and their means are exact: variance 0
        for r, v in ((0, BIG), (1, -BIG)):
            assert mean[r] == v and torch.equal(out[r], b.to(dtype))
            # eps, the root and the quotient rounded
            assert abs(rstd[r].item() - EPS**-0.5) <= 4 * U * EPS**-0.5
    # a row of ordinary values is what it is alone
    alone = torch.empty_like(x[4:])
    pss.pss_layer_norm_forward(x[4:], w, b, EPS, alone)
    assert torch.equal(alone, out[4:])


# widths that leave a part of a group's, a wavefront's or a tile's columns empty,
# inside a vector and not, and widths that fill them
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 5, 12, 64, 100, 101, 512, 520, 1001, 1500, 4100, 5000, 9001, 12304,
                                  16390, 20001, 32768])
def test_backward_of_large_rows(cols, dtype):
    """Constant rows so large that their mean times rstd is beyond float32: their
    z is 0, and g = rstd (h - mean(h)), whatever the width."""
    rng = np.random.default_rng(cols)
    s, dy = make_rows(rng, 4, cols, dtype, 1.5, 0.4), make_rows(rng, 4, cols, dtype)
    s[0], s[2] = 2.0**120, -2.0**120
    w = make_rows(rng, 1, cols, F32, 0.3, 1.0)[0]
    _, mean, rstd = ro.layer_norm(numpy64(s), None, None, EPS)
    mean, rstd = (torch.from_numpy(v).float().cuda() for v in (mean, rstd))
    gx, gw, gb = torch.empty_like(s), *(torch.empty(cols, device="cuda") for _ in range(2))
    pss.pss_layer_norm_backward(dy, s, w, mean, rstd, gx, gw, gb)
    ref, tol = norm_grad_ref(numpy64(dy), numpy64(s), numpy64(w), numpy64(mean), numpy64(rstd), None,
                             None, 1.0, dtype, 4)
    for got, i, what in ((gx, 0, "grad_x"), (gw, 2, "grad_weight"), (gb, 3, "grad_bias")):
        assert bool(got.isfinite().all()), what
        within(got, ref[i], tol[i], what)
