"""Results of more than 64 MB, which are stored past the caches by kernels of
their own and walked over differently: sampled rows against the float64
definitions, and whole arrays against the same calls in smaller parts."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss
from rows_common import EPS, make_drop, norm_ref, numpy64, rounded, sum_ref, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# group of lanes, spans, block, wide form; whole vectors and not
COLS = [1, 5, 8, 16, 37, 64, 100, 128, 500, 511, 520, 1000, 1001, 2048, 2051, 4096, 5000, 9001, 16384, 20003]


def _rows(cols, dtype):
    return (68 << 20) // (cols * (4 if dtype is F32 else 2)) + 3


def _samples(rows):
    n = min(6, rows)
    return sorted({0, 1, rows // 2, max(0, rows - n)}), n


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", COLS)
def test_dropout_and_norm(cols, dtype):
    rows = _rows(cols, dtype)
    g = torch.Generator("cuda").manual_seed(cols)
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    w, b = (torch.randn(cols, generator=g, device="cuda") for _ in range(2))
    drop = make_drop(0.25)
    out, total = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    mean, rstd = (torch.full((rows,), -7.0, device="cuda") for _ in range(2))
    where, n = _samples(rows)

    def kept(r0):
        return ro.mask(drop.p, drop.seed, drop.offset, n, cols, r0)

    for residual in (None, r):
        out.fill_(7.0)
        pss.pss_dropout(x, drop, out, residual=residual)
        for r0 in where:
            s, err = sum_ref(numpy64(x[r0:r0 + n]), None if residual is None else
                             numpy64(r[r0:r0 + n]), *kept(r0))
            within(out[r0:r0 + n], s, rounded(s, err, dtype), ("dropout", r0))
    for residual, d in ((None, None), (r, drop)):
        out.fill_(7.0)
        total.fill_(7.0)
        pss.pss_layer_norm_forward(x, w, b, EPS, out, mean, rstd, residual=residual, dropout=d,
                                   sum_out=total)
        for r0 in where:
            k, scale = kept(r0) if d is not None else (None, 1.0)
            s, err = sum_ref(numpy64(x[r0:r0 + n]), None if residual is None else
                             numpy64(r[r0:r0 + n]), k, scale)
            ref, tol = norm_ref(s, err, numpy64(w), numpy64(b), EPS, dtype)
            for got, want, t, what in zip((out, mean, rstd), ref, tol, ("out", "mean", "rstd")):
                within(got[r0:r0 + n], want, t, (what, r0))
            within(total[r0:r0 + n], s, rounded(s, err, dtype), ("sum", r0))
        # a row that no group took would have kept its filling
        assert bool((rstd > 0).all())
        assert not bool((total == 7.0).all(1).any()) or cols == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [8, 37, 128, 520, 1001, 4096])
def test_norm_equals_its_parts(cols, dtype):
    rows = _rows(cols, dtype)
    x = torch.randn(rows, cols, device="cuda").to(dtype)
    w = torch.randn(cols, device="cuda")
    out, parts = torch.empty_like(x), torch.empty_like(x)
    pss.pss_layer_norm_forward(x, w, None, EPS, out)
    for a, b in zip(x.split(rows // 3), parts.split(rows // 3)):
        pss.pss_layer_norm_forward(a, w, None, EPS, b)
    assert torch.equal(out, parts)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,Q,K", [(8, 1, 4096), (8, 3, 1001), (4, 20, 20), (4, 33, 65), (2, 64, 517),
                                   (2, 300, 520), (1, 512, 2048), (1, 257, 4099), (3, 9, 7), (1, 100, 516)])
def test_bias_equals_its_parts(H, Q, K, dtype):
    m = pss.make_position_buckets(32, 128, True)
    B = (68 << 20) // (H * Q * K * (4 if dtype is F32 else 2)) + 4
    table = torch.randn(32, H, device="cuda")
    x = torch.randn(B, H, Q, K, device="cuda").to(dtype)
    starts = torch.arange(B, dtype=torch.int32, device="cuda") % K
    out, parts = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    pss.pss_position_bias_forward(table, m, out, scores=x, q_starts=starts)
    n = -(-B // 3)
    for a, b, s in zip(x.split(n), parts.split(n), starts.split(n)):
        pss.pss_position_bias_forward(table, m, b, scores=a, q_starts=s)
    assert torch.equal(out, parts)
    b = B - 1
    buckets = ro.bucket_matrix(int(starts[b]), Q, K, lambda d: ro.bucket(d, 32, 128, True))[None]
    ref = ro.position_bias(numpy64(table), buckets, numpy64(x[b:]))
    within(out[b:], ref, rounded(ref, 2.0**-24 * np.abs(ref), dtype), "last")
