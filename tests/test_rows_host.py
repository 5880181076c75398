"""Dropout masks, layer norm and the relative position bias on the host: the
generator against its published vectors, the buckets against integer powers,
the oracle's gradients against differences, and every refusal."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss

D = ctypes.c_void_p(0x1000)  # never dereferenced: checks fail before any use
OK, INVALID, UNSUPPORTED = pss.PSS_OK, pss.PSS_ERR_INVALID_ARG, pss.PSS_ERR_UNSUPPORTED


# (counter, key) -> words, Philox4x32-10's published known answers
KNOWN = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,words", KNOWN)
def test_generator_known_answers(counter, key, words):
    assert tuple(ro.philox4x32(counter, key)) == words


def test_numbers_are_the_generators_halves():
    seed, n = 0x299F31D0A4093822, 0x0370734413198A2E
    got = ro.numbers(seed, n, 1, 16, row0=5)
    for piece in range(2):
        w = ro.philox4x32((piece, 5, n & 0xFFFFFFFF, n >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        for u in range(8):
            assert got[0, piece * 8 + u] == (w[u // 2] >> (16 * (u % 2))) & 0xFFFF


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.25, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("rows,cols,row0", [(3, 1, 0), (5, 17, 2**20), (2, 64, 2**31 - 3)])
def test_mask_matches_oracle(p, rows, cols, row0):
    seed, n = 2**63 + 12345, 2**40 + 7
    got = pss.pss_dropout_mask_host(pss.make_dropout_params(p, seed, n), rows, cols, row0)
    kept, _ = ro.mask(p, seed, n, rows, cols, row0)
    assert np.array_equal(got.astype(bool), kept)


def test_mask_pins_every_number():
    """Thresholds just at and just above a number: the mask flips there."""
    num = ro.numbers(9, 1, 2, 24)
    for r in range(2):
        for c in range(24):
            for t, keep in ((num[r, c], 1), (num[r, c] + 1, 0)):
                d = pss.make_dropout_params(t / 65536, 9, 1)
                assert pss.pss_dropout_mask_host(d, 2, 24)[r, c] == keep


def test_mask_share_and_independence():
    """Of 2^18 elements the dropped share is within 6 standard deviations of p;
    masks of neighbouring numbers, seeds and rows agree as often as
    independent ones."""
    p, n = 0.3, 1 << 18
    t = ro.threshold(p) / 65536
    masks = [ro.mask(p, s, o, 256, n // 256)[0] for s, o in ((1, 0), (1, 1), (2, 0))]
    sd = np.sqrt(t * (1 - t) / n)
    for m in masks:
        assert abs((~m).mean() - t) < 6 * sd
    agree = t * t + (1 - t) ** 2
    sd = np.sqrt(agree * (1 - agree) / n)
    for a, b in ((masks[0], masks[1]), (masks[0], masks[2]), (masks[0][:-1], masks[0][1:])):
        assert abs((a == b).mean() - agree) < 6.2 * sd


@pytest.mark.parametrize("num,far,both", [(32, 128, True), (32, 128, False), (64, 64, False),
                                          (8, 5, True), (4, 2, True), (2, 2, False),
                                          (256, 1000, True), (6, 2**31 - 1, False),
                                          (256, 257, False), (10, 81, True)])
def test_buckets_match_integer_powers(num, far, both):
    m = pss.make_position_buckets(num, far, both)
    n = np.unique(np.concatenate([np.arange(-300, 301), [-far, -far - 1, far - 1, far, far + 1],
                                  np.geomspace(1, 2**31, 40).astype(np.int64),
                                  -np.geomspace(1, 2**31, 40).astype(np.int64)]))
    side = num // 2 if both else num
    borders = np.array(m.borders[:side])
    n = np.concatenate([n, borders - 1, borders, borders + 1])
    want = [ro.bucket(int(v), num, far, both) for v in n]
    assert np.array_equal(pss.pss_position_buckets_host(m, n), want)
    assert pss.pss_position_buckets_host(m, [-2**63])[0] == (num - 1 if both else 0)


def test_buckets_of_own_borders():
    """A program's own map: repeated borders leave buckets empty."""
    m = pss.pss_position_buckets(6, 1)
    m.borders[:3] = [0, 0, 4]
    assert list(pss.pss_position_buckets_host(m, [0, 3, 4, -1, -3, -4])) == [1, 1, 2, 4, 4, 5]
    m = pss.pss_position_buckets(1, 0)
    assert list(pss.pss_position_buckets_host(m, [-5, 0, 5])) == [0, 0, 0]


def test_usual_buckets():
    """32 buckets to distance 128 in both directions: 8 distances of their own,
    then the steps 8 * 2^(j/2)."""
    m = pss.make_position_buckets(32, 128, True)
    assert list(m.borders[:16]) == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


def test_oracle_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    s, w, b = rng.normal(1, 2, (3, 7)), rng.normal(1, 0.3, 7), rng.normal(0, 1, 7)
    dy = rng.normal(0, 1, (3, 7))
    _, mean, rstd = ro.layer_norm(s, w, b, 1e-5)
    g, gw, gb = ro.layer_norm_grad(dy, s, w, mean, rstd)

    def loss(s, w, b):
        return (ro.layer_norm(s, w, b, 1e-5)[0] * dy).sum()

    # central differences of step 1e-5: truncation ~1e-10 of the third
    # derivatives, rounding ~1e-16 / 1e-5
    for arg, grad in ((0, g), (1, gw), (2, gb)):
        for at in np.ndindex(grad.shape):
            v = [s.copy(), w.copy(), b.copy()]
            v[arg][at] += 1e-5
            hi = loss(*v)
            v[arg][at] -= 2e-5
            assert abs((hi - loss(*v)) / 2e-5 - grad[at]) < 1e-7


def test_oracle_bias_gradient_is_the_transpose():
    rng = np.random.default_rng(2)
    of = lambda n: ro.bucket(n, 8, 9, True)  # noqa: E731
    buckets = np.stack([ro.bucket_matrix(f, 5, 11, of) for f in (0, 4)])
    table, dy = rng.normal(size=(8, 3)), rng.normal(size=(2, 3, 5, 11))
    got = (ro.position_bias_grad(dy, buckets, 8) * table).sum()
    assert abs((ro.position_bias(table, buckets) * dy).sum() - got) < 1e-12


# ---- refusals through the C ABI ------------------------------------------------


def _drop(p=0.1):
    d = pss.pss_dropout_params()
    d.p = p
    return d


def _rows(rows=4, cols=16, dtype=0, weight_dtype=0):
    return pss.pss_rows_params(rows, cols, dtype, weight_dtype)


def _dropout(params=None, drop="default", x=D, xs=16, res=None, rs=0, out=D, os_=16):
    d = _drop() if drop == "default" else drop
    p = _rows() if params is None else params
    return pss.load_library().pss_dropout(ctypes.byref(p), None if d is None else ctypes.byref(d), x,
                                          xs, res, rs, out, os_, None)


@pytest.mark.parametrize("kw", [
    dict(params=_rows(rows=-1)), dict(params=_rows(rows=2**31)), dict(params=_rows(cols=0)),
    dict(params=_rows(cols=2**30 + 1)), dict(drop=None), dict(drop=_drop(-0.1)),
    dict(drop=_drop(1.1)), dict(drop=_drop(float("nan"))), dict(x=None), dict(out=None),
    dict(xs=-1), dict(os_=15), dict(res=D, rs=-16), dict(xs=2**47), dict(os_=2**62)])
def test_dropout_refuses(kw):
    assert _dropout(**kw) == INVALID


def test_dropout_refuses_unknown_types_and_takes_no_rows():
    assert _dropout(params=_rows(dtype=2)) == UNSUPPORTED
    assert _dropout(params=_rows(rows=0), x=None, out=None) == OK


def _forward(params=None, drop=None, x=D, xs=16, res=None, w=D, b=D, eps=1e-5, out=D, os_=16,
             sum_=None, ss=16):
    p = _rows() if params is None else params
    return pss.load_library().pss_layer_norm_forward(
        ctypes.byref(p), None if drop is None else ctypes.byref(drop), x, xs, res, 16, w, b, eps, out,
        os_, sum_, ss, None, None, None)


@pytest.mark.parametrize("kw", [
    dict(params=_rows(cols=0)), dict(params=_rows(rows=-1)), dict(drop=_drop(2.0)), dict(x=None),
    dict(out=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")),
    dict(xs=-1), dict(os_=8), dict(sum_=ctypes.c_void_p(0x9000), ss=8), dict(sum_=D)])
def test_norm_forward_refuses(kw):
    assert _forward(**kw) == INVALID


def test_norm_forward_refuses_unknown_types_and_takes_no_rows():
    assert _forward(params=_rows(dtype=-1)) == UNSUPPORTED
    assert _forward(params=_rows(weight_dtype=5)) == UNSUPPORTED
    assert _forward(params=_rows(rows=0, weight_dtype=5), w=None, b=None, x=None, out=None) == OK


def _backward(params=None, drop=None, g=D, gs=16, s=D, w=D, mean=D, rstd=D, up=None, gx=D, gxs=16,
              gr=None, grs=16, gw=D, gb=None):
    p = _rows() if params is None else params
    return pss.load_library().pss_layer_norm_backward(
        ctypes.byref(p), None if drop is None else ctypes.byref(drop), g, gs, s, 16, w, mean, rstd, up,
        -1, gx, gxs, gr, grs, gw, gb, None)


@pytest.mark.parametrize("kw", [
    dict(params=_rows(cols=0)), dict(drop=_drop(-1.0)), dict(g=None), dict(s=None), dict(mean=None),
    dict(rstd=None), dict(gs=-16), dict(up=D), dict(gxs=4), dict(gr=ctypes.c_void_p(0x9000), grs=15),
    dict(gr=D), dict(gb=D), dict(gx=None, gw=None)])
def test_norm_backward_refuses(kw):
    assert _backward(**kw) == INVALID


def test_norm_backward_refuses_unknown_types():
    assert _backward(params=_rows(dtype=9)) == UNSUPPORTED
    assert _backward(params=_rows(weight_dtype=9)) == UNSUPPORTED
    assert _backward(params=_rows(rows=0), gw=None) == OK


@pytest.mark.parametrize("a", [(1, 128, 0), (257, 1000, 0), (2, 128, 1), (9, 128, 1), (32, 8, 1),
                               (32, 16, 0), (32, 0, 1), (32, -5, 0), (32, 128, 2)])
def test_buckets_refuse(a):
    lib, m = pss.load_library(), pss.pss_position_buckets(7, 0)
    assert lib.pss_position_buckets_init(*a, ctypes.byref(m)) == INVALID
    assert m.num_buckets == 7  # untouched
    assert lib.pss_position_buckets_init(32, 128, 1, None) == INVALID


def _scores(B=2, H=3, Q=4, K=5, dtype=0, table=0, start=0, ins=None, outs=None):
    three = ctypes.c_int64 * 3
    dense = (H * Q * K, Q * K, K)
    return pss.pss_scores_params(B, H, Q, K, dtype, table, start, three(*(ins or dense)),
                                 three(*(outs or dense)))


def _map(num=8, both=1, **borders):
    m = pss.make_position_buckets(8, 64, True)
    m.num_buckets, m.bidirectional = num, both
    for i, v in borders.items():
        m.borders[int(i[1:])] = v
    return m


BAD_BIAS = [
    dict(p=_scores(B=-1)), dict(p=_scores(H=-1)), dict(p=_scores(B=2**16, H=2**15)),
    dict(p=_scores(Q=-1)), dict(p=_scores(Q=2**29 + 1)), dict(p=_scores(K=-1)),
    dict(p=_scores(K=2**30 + 1)), dict(p=_scores(start=-1)), dict(p=_scores(start=2**29 + 1)),
    dict(p=_scores(ins=(60, 20, -5))), dict(p=_scores(ins=(2**60, 20, 5))), dict(m=None),
    dict(m=_map(num=0)), dict(m=_map(num=257)), dict(m=_map(num=7)), dict(m=_map(both=2)),
    dict(m=_map(i0=1)), dict(m=_map(i2=0)), dict(m=_map(i1=-1)), dict(p=None)]


def _bias(p=_scores(), m=_map(), table=D, scores=D, out=D):
    return pss.load_library().pss_position_bias_forward(
        None if p is None else ctypes.byref(p), None if m is None else ctypes.byref(m), table, None,
        scores, out, None)


def _bias_back(p=_scores(), m=_map(), g=D, gt=D):
    return pss.load_library().pss_position_bias_backward(
        None if p is None else ctypes.byref(p), None if m is None else ctypes.byref(m), None, g, gt,
        None)


@pytest.mark.parametrize("kw", BAD_BIAS)
def test_bias_refuses(kw):
    assert _bias(**kw) == INVALID
    assert _bias_back(**kw) == INVALID


def test_bias_refuses_null_overlap_and_types():
    assert _bias(table=None) == INVALID
    assert _bias(out=None) == INVALID
    for outs in ((60, 20, 4), (60, 19, 5), (59, 20, 5), (0, 20, 5)):
        assert _bias(p=_scores(outs=outs)) == INVALID
    assert _bias(p=_scores(dtype=2)) == UNSUPPORTED
    assert _bias(p=_scores(table=2)) == UNSUPPORTED
    assert _bias(p=_scores(B=2**30, H=1, Q=2**20, K=2**20)) == UNSUPPORTED
    assert _bias_back(g=None) == INVALID
    assert _bias_back(gt=None) == INVALID
    assert _bias_back(p=_scores(dtype=2)) == UNSUPPORTED
    for empty in (dict(B=0), dict(H=0), dict(Q=0), dict(K=0)):
        assert _bias(p=_scores(**empty), table=None, scores=None, out=None) == OK
    assert _bias_back(p=_scores(H=0), g=None, gt=None) == OK


def test_host_forms_refuse():
    lib = pss.load_library()
    buf, n = (ctypes.c_uint8 * 64)(), (ctypes.c_int64 * 1)(0)
    ok = _drop()
    f = lib.pss_dropout_mask_host
    for a in [(None, 0, 1, 8, buf), (ctypes.byref(_drop(3.0)), 0, 1, 8, buf),
              (ctypes.byref(ok), -1, 1, 8, buf), (ctypes.byref(ok), 0, -1, 8, buf),
              (ctypes.byref(ok), 2**31 - 1, 1, 8, buf), (ctypes.byref(ok), 0, 1, 0, buf),
              (ctypes.byref(ok), 0, 1, 8, None)]:
        assert f(*a) == INVALID
    g = lib.pss_position_buckets_host
    m = _map()
    assert g(None, n, 1, buf) == INVALID
    assert g(ctypes.byref(m), None, 1, buf) == INVALID
    assert g(ctypes.byref(m), n, 1, None) == INVALID
    assert g(ctypes.byref(m), n, -1, buf) == INVALID
    assert g(ctypes.byref(m), None, 0, None) == OK


# ---- refusals of the binding (CPU tensors: before anything is enqueued) -----------


def test_binding_refuses_cpu_tensors_and_wrong_types():
    x, d = torch.zeros(4, 8), pss.make_dropout_params(0.1, 1)
    m = pss.make_position_buckets(8, 64, True)
    with pytest.raises(ValueError):
        pss.pss_dropout(x, d, x)
    with pytest.raises(TypeError):
        pss.pss_dropout(x.double(), d, x.double())
    with pytest.raises(ValueError):
        pss.pss_layer_norm_forward(x, None, None, 1e-5, x)
    with pytest.raises(ValueError):
        pss.pss_layer_norm_backward(x, x, None, None, None, x)
    with pytest.raises(ValueError):
        pss.pss_position_bias_forward(torch.zeros(8, 3), m, torch.zeros(2, 3, 4, 5))
    with pytest.raises(TypeError):
        pss.pss_position_bias_backward(torch.zeros(2, 3, 4, 5).half(), m, torch.zeros(8, 3))
    with pytest.raises(ValueError):
        pss.make_dropout_params(1.5, 1)
    with pytest.raises(ValueError):
        pss.make_dropout_params(float("nan"), 1)
    with pytest.raises(TypeError):
        pss.make_dropout_params(0.5, 1, step=torch.zeros(1))
    with pytest.raises(ValueError):
        pss.make_dropout_params(0.5, 1, step=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(pss.PssError):
        pss.make_position_buckets(3, 128, True)
