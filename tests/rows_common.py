"""Inputs, float64 references and derived error bounds of the row operators'
GPU tests.

u = 2^-24 is a float32 rounding, HALF[type] the rounding of the result's
type.  A sum of n float32 terms in any order is off by at most n u times the
sum of their magnitudes; the kernels sum a row in lanes and then across them,
so CHAIN(cols) additions bound the longest chain of one row's sum.
"""
import numpy as np
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss

U = 2.0**-24
HALF = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8}
EPS = 1e-5


def chain(cols):
    """Additions on the longest path of one row's sum: a lane's own elements
    (64 lanes at least share a row of more than 512 elements; 8 elements to a
    lane below that) and two trees."""
    return max(8, -(-cols // 64)) + 24


def numpy64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def make_rows(rng, rows, cols, dtype, scale=1.0, shift=0.0, pad=0, dev="cuda"):
    """[rows][cols] view of rows `pad` elements longer (the rest is NaN)."""
    wide = np.full((rows, cols + pad), np.nan)
    wide[:, :cols] = rng.normal(shift, scale, (rows, cols))
    return torch.from_numpy(wide).to(dev, dtype)[:, :cols]


def out_rows(rows, cols, dtype, pad=0, dev="cuda"):
    """A result's rows in a frame of 7s (checked by frame_kept)."""
    return torch.full((rows, cols + pad), 7.0, dtype=dtype, device=dev)[:, :cols]


def frame_kept(view):
    base = view._base
    return base is None or bool((base[:, view.shape[1]:] == 7.0).all())


def within(got, ref, tol, what):
    got = numpy64(got)
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= tol) & ~((got == ref) | (np.isnan(got) & np.isnan(ref)))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3],
                           ref[bad][:3], np.broadcast_to(tol, ref.shape)[bad][:3])


def rounded(ref, err, dtype):
    """Bound of a value within err of ref, rounded to dtype once."""
    return err + HALF[dtype] * (np.abs(ref) + err) + 1e-38


def mask_of(drop, rows, cols, step=0):
    if drop is None:
        return None, 1.0
    return ro.mask(drop.p, drop.seed, (drop.offset + step) % 2**64, rows, cols)


def sum_ref(x, residual, kept, scale):
    """s = residual + D(x) and the error of its float32 value: the rounded
    scale, the product and the sum."""
    s = ro.dropout(x, kept, scale)
    err = (2 * U * np.abs(s)) if kept is not None else np.zeros_like(s)
    if residual is not None:
        s = s + residual
        err = err + U * (np.abs(s) + err)
    return s, err


def norm_ref(s, s_err, weight, bias, eps, dtype):
    """(out, mean, rstd) in float64 and their bounds: with A the mean magnitude
    of a row, the mean is off by (chain + 2) u A + the mean of s_err; a
    difference from it by d; the variance v = sum e^2 / C by 2 d mean|e| + d^2
    + chain u v, hence 1/sqrt(v + eps) by half of that relative to v + eps
    (first order; doubled here for the rest)."""
    C = s.shape[1]
    k = chain(C) + 4
    w = np.ones(C) if weight is None else weight
    b = np.zeros(C) if bias is None else bias
    out, mean, rstd = ro.layer_norm(s, weight, bias, eps)
    e = s - mean[:, None]
    mean_err = k * U * np.abs(s).mean(1) + s_err.mean(1)
    d = mean_err[:, None] + s_err + U * (np.abs(e) + mean_err[:, None])
    v = (e * e).mean(1) + eps
    v_err = (2 * np.abs(e) * d + d * d).mean(1) + (k + 4) * U * v
    rel = v_err / v + 4 * U
    z = np.abs(e) * rstd[:, None]
    err = np.abs(w) * (d * rstd[:, None] * (1 + rel[:, None]) + z * (rel[:, None] + 4 * U)) \
        + 2 * U * (np.abs(w) * z + np.abs(b))
    return (out, mean, rstd), (rounded(out, err, dtype), mean_err + U * np.abs(mean) + 1e-38,
                               rstd * rel)


def norm_grad_ref(dy, s, weight, mean, rstd, up, kept, scale, dtype, row_chain):
    """((grad_x, grad_residual, grad_weight, grad_bias), bounds).  z has two
    roundings and the difference's own; the two sums are off by chain u times
    their magnitudes; the last line adds four more products and sums."""
    C = s.shape[1]
    k = chain(C) + 10
    g, gw, gb = ro.layer_norm_grad(dy, s, weight, mean, rstd)
    z = np.abs((s - mean[:, None]) * rstd[:, None])
    h = np.abs(dy * (1 if weight is None else weight))
    err = k * U * rstd[:, None] * (h + h.mean(1, keepdims=True)
                                   + z * (h * z).mean(1, keepdims=True))
    if up is not None:
        g = g + up
        err = err + U * (np.abs(g) + np.abs(up))
    gx = ro.dropout(g, kept, scale)
    ex = err if kept is None else np.where(kept, err * scale + 2 * U * np.abs(gx), 0.0)
    kr = row_chain + 6
    return (gx, g, gw, gb), (rounded(gx, ex, dtype), rounded(g, err, dtype),
                             kr * U * (np.abs(dy) * z).sum(0) + 1e-38,
                             kr * U * np.abs(dy).sum(0) + 1e-38)


def row_chain(rows):
    """Additions on the longest path of a sum over rows: a block's own rows
    (at least 64 blocks share more than 64 rows) and the parts of at most 1024
    blocks."""
    return min(rows, -(-rows // 64) + 1024)


def make_drop(p, seed=77, offset=3, step=None):
    return None if p is None else pss.make_dropout_params(p, seed, offset, step)
