"""Operators on rows and the position bias where a call needs more workgroups
than one grid dimension holds (2^32 work-items): every element is written."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss
from rows_common import EPS, U, make_drop, numpy64, rounded, sum_ref, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _need(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2**30:
        pytest.skip(f"needs {gib} GiB of GPU memory")


def test_dropout_of_more_rows_than_one_grid_dimension():
    """2^26 + 5 rows of 257 (4 to a workgroup: 2^24 + 2 of them), one input row
    for all."""
    _need(70)
    rows, cols = 2**26 + 5, 257
    x = torch.linspace(1, 2, cols, device="cuda").to(BF16)[None]
    out = torch.full((rows, cols), 7.0, dtype=BF16, device="cuda")
    drop = make_drop(0.25)
    pss.pss_dropout(x.expand(rows, cols), drop, out)
    xin = numpy64(x)
    for r0 in (0, 2**25 - 1, 2**26 - 3, rows - 40):
        kept = ro.mask(drop.p, drop.seed, drop.offset, 40 if r0 + 40 <= rows else rows - r0, cols, r0)[0]
        s, err = sum_ref(np.broadcast_to(xin, kept.shape), None, kept, 65536 / (65536 - 16384))
        within(out[r0:r0 + kept.shape[0]], s, rounded(s, err, BF16), r0)
    for part in out.split(2**24):  # a kept element is at most 8 / 3
        assert bool((part < 3).all())


@pytest.mark.parametrize("Q,K,B,H", [(4, 20, 2**22 + 3, 17), (33, 129, 2**16 + 1, 64),
                                     (9, 33, 2**20 + 1, 65)])
def test_bias_of_more_scores_than_one_grid_dimension(Q, K, B, H):
    """The bias alone, the same for every sequence; short rows, several to a
    workgroup."""
    _need(50)
    m = pss.make_position_buckets(32, 128, True)
    table = torch.randn(32, H, device="cuda")
    out = torch.full((B, H, Q, K), 900.0, dtype=BF16, device="cuda")
    pss.pss_position_bias_forward(table, m, out, q_start=3)
    buckets = ro.bucket_matrix(3, Q, K, lambda n: ro.bucket(n, 32, 128, True))[None]
    ref = ro.position_bias(numpy64(table), buckets)
    within(out[:1], ref, rounded(ref, 0, BF16), "first")
    for part in out.split(2**16):
        assert bool((part == out[:1]).all())


def test_far_gradient_of_more_tiles_than_one_grid_dimension():
    """2^22 + 5 sequences that share one gradient (its sum is exact: powers of
    two), borders beyond the near form's."""
    m = pss.pss_position_buckets(2, 0)
    m.borders[:2] = [0, 5000]
    B, Q, K = 2**22 + 5, 8, 20
    g = torch.zeros(1, 1, Q, K, device="cuda")
    g[0, 0, 0, 3] = 1.0
    out = torch.full((2, 1), 7.0, device="cuda")
    pss.pss_position_bias_backward(g.expand(B, 1, Q, K), m, out, q_start=5002)
    # query 0 is 5002 - 3 = 4999 from its key: below the border
    assert out.tolist() == [[float(B)], [0.0]]


def test_norm_backward_of_more_columns_than_one_grid_holds():
    """One row of 2^26 + 3 columns: 2^23 workgroups' worth of column sums."""
    _need(40)
    cols = 2**26 + 3
    s = torch.randn(1, cols, device="cuda", dtype=BF16)
    dy = torch.randn(1, cols, device="cuda", dtype=BF16)
    mean, rstd = s.double().mean(1).float(), (s.double().var(1, correction=0) + EPS).rsqrt().float()
    gw, gb = (torch.full((cols,), 7.0, device="cuda") for _ in range(2))
    gx = torch.empty_like(s)
    pss.pss_layer_norm_backward(dy, s, None, mean, rstd, gx, gw, gb)
    z = (s.double() - mean.double()) * rstd.double()
    d = dy.double()
    assert torch.equal(gb, dy[0].float())
    assert bool(((gw - (d * z)[0]).abs() <= 4 * U * (d * z)[0].abs() + 2 * U * d[0].abs() + 1e-38).all())
    g = rstd.double() * (d - d.mean() - z * (d * z).mean())
    # the two means: 2^15 pieces of 8 to a lane, so 2^15 + 40 additions at most
    err = (2**15 + 40) * U * rstd.double() * (d.abs().mean() + z.abs() * (d * z).abs().mean())
    err += 10 * U * rstd.double() * (d.abs() + z.abs())
    assert bool(((gx.double() - g).abs() <= err + 2.0**-8 * (g.abs() + err)).all())
