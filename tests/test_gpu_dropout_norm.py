"""Dropout and layer norm (forward, backward) on the GPU against the float64
definitions, through the binding."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss
from rows_common import (EPS, HALF, U, chain, frame_kept, make_drop, make_rows, mask_of, norm_grad_ref,
                         norm_ref, numpy64, out_rows, rounded, row_chain, sum_ref, within)

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (3, 1), (5, 2), (1, 7), (70, 8), (9, 9), (300, 16), (37, 63), (130, 64), (33, 65),
          (257, 128), (19, 129), (40, 255), (21, 512), (13, 520), (11, 1000), (17, 1001), (6, 2048),
          (5, 2051), (7, 4096), (3, 4100), (4, 8192), (2, 8200), (3, 16384), (2, 20001), (1, 40000)]


def _check_dropout(x, residual, out, drop, step=0):
    kept, scale = mask_of(drop, *x.shape, step)
    xin, rin, dt = numpy64(x), numpy64(residual), x.dtype
    pss.pss_dropout(x, drop, out, residual=residual)
    s, err = sum_ref(xin, rin, kept, scale)
    within(out, s, rounded(s, err, dt), "out")
    assert frame_kept(out)
    if residual is None:  # the zeros are the mask's
        got = numpy64(out)
        assert np.array_equal(got != 0, kept & (xin != 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dropout(rows, cols, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    for p, pad, res in ((0.1, 0, False), (0.5, 3, True), (0.0, 5, True)):
        x = make_rows(rng, rows, cols, dtype, 2.0, 0.3, pad)
        r = make_rows(rng, rows, cols, dtype, 1.0, 0.0, 2 * pad) if res else None
        _check_dropout(x, r, out_rows(rows, cols, dtype, pad), make_drop(p, offset=2**40 + cols))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_extremes(dtype):
    """p = 1 drops everything (infinities and NaN too), p below 2^-17 nothing;
    a dropped infinity is 0, a kept one stays."""
    x = torch.full((4, 100), float("inf"), dtype=dtype, device="cuda")
    x[1] = float("nan")
    x[2] = torch.finfo(dtype).min
    out = torch.empty_like(x)
    pss.pss_dropout(x, make_drop(1.0), out)
    assert bool((out == 0).all())
    pss.pss_dropout(x, make_drop(2.0**-18), out)
    assert torch.equal(out.nan_to_num(5.0), x.nan_to_num(5.0))
    d = make_drop(0.25)
    kept, _ = mask_of(d, 4, 100)
    pss.pss_dropout(x, d, out)
    got = numpy64(out)
    assert (got[~kept] == 0).all() and np.isinf(got[0][kept[0]]).all()
    assert np.isnan(got[1][kept[1]]).all()


def test_dropout_in_place_and_broadcast():
    rng = np.random.default_rng(5)
    d = make_drop(0.3)
    kept, scale = mask_of(d, 50, 77)
    for into in ("x", "residual"):
        x, r = make_rows(rng, 50, 77, F32), make_rows(rng, 50, 77, F32)
        s, err = sum_ref(numpy64(x), numpy64(r), kept, scale)
        out = x if into == "x" else r
        pss.pss_dropout(x, d, out, residual=r)
        within(out, s, rounded(s, err, F32), into)
    x, r = make_rows(rng, 50, 77, F32), make_rows(rng, 1, 77, F32).expand(50, 77)
    _check_dropout(x, r, torch.empty(50, 77, device="cuda"), d)  # one residual row for all


def test_dropout_gradient_is_the_same_mask():
    """The gradient of sum(out * g) is D(g): elementwise, against differences of
    the forward call itself (linear in x: exact up to rounding)."""
    rng = np.random.default_rng(6)
    d = make_drop(0.4)
    x, g = make_rows(rng, 20, 33, F32), make_rows(rng, 20, 33, F32)
    grad, lo, hi = (torch.empty(20, 33, device="cuda") for _ in range(3))
    pss.pss_dropout(g, d, grad)
    pss.pss_dropout(x - 1, d, lo)
    pss.pss_dropout(x + 1, d, hi)
    # roundings: x -+ 1 and their products, each within 2 u of 5 * scale
    within(grad, numpy64((hi - lo) / 2 * g), 40 * U * np.abs(numpy64(g)), "gradient")


def test_dropout_rows_beyond_32_bits():
    """Rows that begin past 2^32 elements, in and out."""
    stride, cols = 2**31 + 24, 1000
    base = torch.empty(2 * stride + cols, dtype=BF16, device="cuda")
    x = base.as_strided((3, cols), (stride, 1))
    rng = np.random.default_rng(8)
    x.copy_(make_rows(rng, 3, cols, BF16))
    _check_dropout(x, None, torch.empty((3, cols), dtype=BF16, device="cuda"), make_drop(0.2))
    ref = x.clone()
    pss.pss_dropout(ref, make_drop(0.0), x, residual=ref)
    assert torch.equal(x, ref + ref)


WEIGHTS = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]


def _norm_case(rng, rows, cols, dtype, wdtype, p, pad, res, affine):
    x = make_rows(rng, rows, cols, dtype, 1.5, 0.4, pad)
    r = make_rows(rng, rows, cols, dtype, 1.0, -0.2, pad) if res else None
    w = make_rows(rng, 1, cols, wdtype, 0.3, 1.0)[0] if affine & 1 else None
    b = make_rows(rng, 1, cols, wdtype, 0.5)[0] if affine & 2 else None
    return x, r, w, b, make_drop(p, offset=cols)


def _check_forward(x, r, w, b, drop, pad, with_sum):
    rows, cols, dt = *x.shape, x.dtype
    out = out_rows(rows, cols, dt, pad)
    total = out_rows(rows, cols, dt, 2 * pad) if with_sum else None
    mean, rstd = (torch.empty(rows, device="cuda") for _ in range(2))
    pss.pss_layer_norm_forward(x, w, b, EPS, out, mean, rstd, residual=r, dropout=drop,
                               sum_out=total)
    kept, scale = mask_of(drop, rows, cols)
    s, s_err = sum_ref(numpy64(x), numpy64(r), kept, scale)
    ref, tol = norm_ref(s, s_err, numpy64(w), numpy64(b), EPS, dt)
    for got, want, t, what in zip((out, mean, rstd), ref, tol, ("out", "mean", "rstd")):
        within(got, want, t, what)
    if total is not None:
        within(total, s, rounded(s, s_err, dt), "sum")
        assert frame_kept(total)
    assert frame_kept(out)


@pytest.mark.parametrize("dtype,wdtype", WEIGHTS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_forward(rows, cols, dtype, wdtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    for p, pad, res, affine in ((None, 0, False, 3), (0.1, 3, True, 3), (0.5, 8, False, 1),
                                (None, 5, True, 2), (0.0, 0, False, 0)):
        x, r, w, b, drop = _norm_case(rng, rows, cols, dtype, wdtype, p, pad, res, affine)
        _check_forward(x, r, w, b, drop, pad, res)


@pytest.mark.parametrize("rows,cols", [(5000, 40), (3000, 128), (700, 1024), (600, 4096), (300, 9000),
                                       (20000, 8)])
def test_norm_forward_many_rows(rows, cols):
    rng = np.random.default_rng(cols)
    for dtype in (F32, BF16):
        x, r, w, b, drop = _norm_case(rng, rows, cols, dtype, F32, 0.1, 0, True, 3)
        _check_forward(x, r, w, b, drop, 0, True)


def test_norm_forward_special_rows():
    """Constant rows (variance 0), rows far from 0, huge and tiny ones; rows
    with an infinity or NaN become NaN and leave the others alone."""
    rng = np.random.default_rng(3)
    for cols in (64, 1000, 4096, 33000):
        x = make_rows(rng, 8, cols, F32)
        x[0] = 3.0
        x[1] = 0.0
        x[2] += 1000.0
        x[3] *= 1e15
        x[4] *= 1e-12
        x[5, cols // 2] = float("inf")
        x[6, cols - 1] = float("nan")
        out, clean = torch.empty_like(x), [0, 1, 2, 3, 4, 7]
        pss.pss_layer_norm_forward(x, None, None, EPS, out)
        assert bool(out[5:7].isnan().all())
        s = numpy64(x)[clean]
        ref, tol = norm_ref(s, np.zeros_like(s), None, None, EPS, F32)
        within(out[clean], ref[0], tol[0], cols)


def test_norm_forward_in_place_and_alone():
    """The residual stream updated in place; out over x; no statistics kept."""
    rng = np.random.default_rng(4)
    for cols in (96, 2000, 33001):
        for dtype in (F32, BF16):
            x, r, w, b, drop = _norm_case(rng, 6, cols, dtype, dtype, 0.2, 0, True, 3)
            out, total = (torch.empty(6, cols, dtype=dtype, device="cuda") for _ in range(2))
            pss.pss_layer_norm_forward(x, w, b, EPS, out, residual=r, dropout=drop, sum_out=total)
            x2, r2 = x.clone(), r.clone()
            pss.pss_layer_norm_forward(x2, w, b, EPS, x2, residual=r2, dropout=drop, sum_out=r2)
            assert torch.equal(x2, out) and torch.equal(r2, total)
            x3 = x.clone()
            pss.pss_layer_norm_forward(x3, w, b, EPS, r2, dropout=drop, sum_out=x3)
            pss.pss_layer_norm_forward(x, w, b, EPS, out, dropout=drop, sum_out=total)
            assert torch.equal(r2, out) and torch.equal(x3, total)


def test_norm_of_a_tables_columns():
    """One table's embeddings inside the pooled rows [B][T*d]."""
    rng = np.random.default_rng(9)
    pooled = make_rows(rng, 200, 5 * 24, F32)
    w = make_rows(rng, 1, 24, F32, 0.3, 1.0)[0]
    out = out_rows(200, 5 * 24, F32)
    pss.pss_layer_norm_forward(pooled[:, 48:72], w, None, EPS, out[:, 48:72])
    s = numpy64(pooled[:, 48:72])
    ref, tol = norm_ref(s, np.zeros_like(s), numpy64(w), None, EPS, F32)
    within(out[:, 48:72], ref[0], tol[0], "table")
    assert bool((out[:, :48] == 7).all()) and bool((out[:, 72:] == 7).all())


def _check_backward(rng, rows, cols, dtype, wdtype, p, pad, up, affine, want, spread=1.0):
    s = make_rows(rng, rows, cols, dtype, 1.5 * spread, 0.4, pad)
    dy = make_rows(rng, rows, cols, dtype, 1.0, 0.05, pad)
    u = make_rows(rng, rows, cols, dtype, 0.7, 0.0, 2 * pad) if up else None
    w = make_rows(rng, 1, cols, wdtype, 0.3, 1.0)[0] if affine else None
    drop = make_drop(p, offset=cols)
    _, mean, rstd = ro.layer_norm(numpy64(s), None, None, EPS)
    mean, rstd = (torch.from_numpy(v).float().cuda() for v in (mean, rstd))
    gx = out_rows(rows, cols, dtype, pad) if "x" in want else None
    gr = out_rows(rows, cols, dtype, 2 * pad) if "r" in want else None
    gw = torch.full((cols,), 7.0, device="cuda") if "w" in want else None
    gb = torch.full((cols,), 7.0, device="cuda") if "b" in want else None
    pss.pss_layer_norm_backward(dy, s, w, mean, rstd, gx, gw, gb, grad_sum=u, dropout=drop,
                                grad_residual=gr)
    kept, scale = mask_of(drop, rows, cols)
    ref, tol = norm_grad_ref(numpy64(dy), numpy64(s), numpy64(w), numpy64(mean), numpy64(rstd),
                             numpy64(u), kept, scale, dtype, row_chain(rows))
    for got, r, t, what in zip((gx, gr, gw, gb), ref, tol, ("grad_x", "grad_residual",
                                                            "grad_weight", "grad_bias")):
        if got is not None:
            within(got, r, t, what)
    for v in (gx, gr):
        assert v is None or frame_kept(v)


@pytest.mark.parametrize("dtype,wdtype", WEIGHTS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_backward(rows, cols, dtype, wdtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    for p, pad, up, affine, want in ((None, 0, False, True, "xwb"), (0.1, 3, True, True, "xrwb"),
                                     (0.5, 8, False, False, "xw"), (None, 5, True, True, "r"),
                                     (0.2, 0, False, True, "b")):
        _check_backward(rng, rows, cols, dtype, wdtype, p, pad, up, affine, want)


@pytest.mark.parametrize("rows,cols", [(70000, 8), (9000, 33), (6000, 128), (5000, 500), (2000, 1024),
                                       (1100, 4096), (600, 9001)])
def test_norm_backward_many_rows(rows, cols):
    rng = np.random.default_rng(cols)
    for dtype in (F32, BF16):
        _check_backward(rng, rows, cols, dtype, F32, 0.1, 0, True, True, "xrwb")


def test_norm_backward_without_rows():
    e = torch.empty(0, 24, device="cuda")
    gw, gb = (torch.full((24,), 7.0, device="cuda") for _ in range(2))
    none = torch.empty(0, device="cuda")
    pss.pss_layer_norm_backward(e, e, None, none, none, e, gw, gb)
    assert bool((gw == 0).all()) and bool((gb == 0).all())
    pss.pss_layer_norm_forward(e, gw, gb, EPS, e)
    pss.pss_dropout(e, make_drop(0.5), e)


def test_norm_backward_in_place_and_repeatable():
    """grad_x over grad_out, grad_residual over grad_sum: the same bits; every
    gradient the same bits from call to call."""
    rng = np.random.default_rng(12)
    for rows, cols in ((3000, 64), (500, 1000), (300, 4096), (40, 33001)):
        for dtype in (F32, BF16):
            s, dy, up = (make_rows(rng, rows, cols, dtype) for _ in range(3))
            w = make_rows(rng, 1, cols, dtype, 0.3, 1.0)[0]
            mean, rstd = s.float().mean(1), 1 / (s.float().var(1) + EPS).sqrt()
            drop = make_drop(0.3)
            runs = []
            for way in range(3):
                gw, gb = (torch.empty(cols, device="cuda") for _ in range(2))
                g, q = dy.clone(), up.clone()
                gx, gr = (g, q) if way == 2 else (torch.empty_like(dy) for _ in range(2))
                pss.pss_layer_norm_backward(g, s, w, mean, rstd, gx, gw, gb, grad_sum=q,
                                            dropout=drop, grad_residual=gr)
                runs.append((gx, gr, gw, gb))
            for other in runs[1:]:
                for a, b in zip(runs[0], other):
                    assert torch.equal(a, b), (rows, cols, dtype)


def test_norm_backward_follows_the_forwards_differences():
    """The gradient against central differences of the GPU forward in one
    direction: out is float32, step 2^-7 of a unit direction."""
    rng = np.random.default_rng(13)
    rows, cols, h = 12, 160, 2.0**-7
    x, r, dy, v = (make_rows(rng, rows, cols, F32) for _ in range(4))
    w, b = make_rows(rng, 1, cols, F32, 0.3, 1.0)[0], make_rows(rng, 1, cols, F32)[0]
    drop = make_drop(0.25)
    out, total, gx = (torch.empty_like(x) for _ in range(3))
    mean, rstd = (torch.empty(rows, device="cuda") for _ in range(2))

    def loss(x):
        pss.pss_layer_norm_forward(x, w, b, EPS, out, mean, rstd, residual=r, dropout=drop,
                                   sum_out=total)
        return (numpy64(out) * numpy64(dy)).sum(1)

    diff = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
    loss(x)
    pss.pss_layer_norm_backward(dy, total, w, mean, rstd, gx, dropout=drop)
    got = (numpy64(gx) * numpy64(v)).sum(1)
    # rounding of out: 16 u per element over 2 h (about 1e-3 in all); the third
    # derivative of the normalised row in a direction of length sqrt(cols)
    # times rstd leaves h^2 / 6 * 6 * |dy| |out| < 3e-2
    assert np.abs(diff - got).max() < 0.04


def test_norm_other_stream_and_current_device():
    """Work goes to the given stream; two streams at once keep their scratch
    apart."""
    rng = np.random.default_rng(14)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    data = []
    for _ in range(2):
        s, dy = make_rows(rng, 2000, 512, F32), make_rows(rng, 2000, 512, F32)
        mean, rstd = s.mean(1), 1 / (s.var(1) + EPS).sqrt()
        data.append((dy, s, mean, rstd, torch.empty_like(s), torch.empty(512, device="cuda"),
                     torch.empty(512, device="cuda")))
    want = []
    for dy, s, mean, rstd, gx, gw, gb in data:
        pss.pss_layer_norm_backward(dy, s, None, mean, rstd, gx, gw, gb)
        want.append([t.clone() for t in (gx, gw, gb)])
        for t in (gx, gw, gb):
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(10):
        for st, (dy, s, mean, rstd, gx, gw, gb) in zip((a, b), data):
            pss.pss_layer_norm_backward(dy, s, None, mean, rstd, gx, gw, gb, stream=st)
    torch.cuda.synchronize()
    for w, d in zip(want, data):
        for x, y in zip(w, d[4:]):
            assert torch.equal(x, y)


def test_captured_step_takes_new_masks_and_shares_no_scratch():
    """Two graphs, each a forward and backward with its masks counted on the
    GPU, replayed in turn with eager work between: every replay as the eager
    calls at that count."""
    rng = np.random.default_rng(15)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def state(rows, cols):
        x, r, dy = (make_rows(rng, rows, cols, F32) for _ in range(3))
        w, b = make_rows(rng, 1, cols, F32, 0.3, 1.0)[0], make_rows(rng, 1, cols, F32)[0]
        bufs = [torch.empty_like(x) for _ in range(4)]
        vecs = [torch.empty(n, device="cuda") for n in (rows, rows, cols, cols)]
        return x, r, dy, w, b, bufs, vecs, pss.make_dropout_params(0.2, 5, cols, step)

    def run(st):
        x, r, dy, w, b, (out, total, gx, gr), (mean, rstd, gw, gb), drop = st
        pss.pss_layer_norm_forward(x, w, b, EPS, out, mean, rstd, residual=r, dropout=drop,
                                   sum_out=total)
        pss.pss_layer_norm_backward(dy, total, w, mean, rstd, gx, gw, gb, grad_sum=dy, dropout=drop,
                                    grad_residual=gr)
        return [t.clone() for t in (out, total, gx, gr, mean, rstd, gw, gb)]

    states = [state(300, 256), state(77, 1500)]
    want = []
    for k in range(4):
        step.fill_(k)
        want.append([run(s) for s in states])
    for i in range(2):  # the mask does change with the count
        assert not torch.equal(want[0][i][0], want[1][i][0])
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(run(s))
        graphs.append(g)
    for k in range(4):
        step.fill_(k)
        for i in (0, 1) if k % 2 else (1, 0):
            graphs[i].replay()
            run(states[1 - i])  # eager work in between
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(outs[i], want[k][i]):
                assert torch.equal(a, b), (k, i)
    kept0, scale = mask_of(make_drop(0.2, 5, 256), 300, 256, 3)
    s, err = sum_ref(numpy64(states[0][0]), numpy64(states[0][1]), kept0, scale)
    within(want[3][0][1], s, rounded(s, err, F32), "mask of count 3")


def test_binding_refuses():
    x = torch.zeros(4, 16, device="cuda")
    v, d = torch.zeros(16, device="cuda"), make_drop(0.1)
    m = torch.zeros(4, device="cuda")
    wide = torch.zeros(4, 32, device="cuda")
    bad_out = [x[:3], x[:, :8], x.bfloat16(), x.cpu(), wide[:, ::2], x[:1].expand(4, 16), v]
    for out in bad_out:
        with pytest.raises((ValueError, TypeError)):
            pss.pss_dropout(x, d, out)
        with pytest.raises((ValueError, TypeError)):
            pss.pss_layer_norm_forward(x, v, v, EPS, out)
        with pytest.raises((ValueError, TypeError)):
            pss.pss_layer_norm_backward(x, x, v, m, m, out)
    for w in (v[:8], v.half(), v.cpu(), wide[0, ::2]):
        with pytest.raises((ValueError, TypeError)):
            pss.pss_layer_norm_forward(x, w, None, EPS, torch.empty_like(x))
        with pytest.raises((ValueError, TypeError)):
            pss.pss_layer_norm_backward(x, x, w, m, m, torch.empty_like(x))
        with pytest.raises((ValueError, TypeError)):
            pss.pss_layer_norm_backward(x, x, v, m, m, torch.empty_like(x), grad_weight=w)
    with pytest.raises(TypeError):
        pss.pss_layer_norm_forward(x, v, v.bfloat16(), EPS, torch.empty_like(x))
    with pytest.raises(ValueError):
        pss.pss_layer_norm_backward(x, x, v, m, None, torch.empty_like(x))
    with pytest.raises(ValueError):
        pss.pss_dropout(x, None, x)
    with pytest.raises(pss.PssError):
        pss.pss_layer_norm_forward(x, v, v, 0.0, torch.empty_like(x))
    with pytest.raises(pss.PssError):
        pss.pss_layer_norm_backward(x, x, v, m, m, None)
    assert HALF[F32] == U and chain(8) == 32
