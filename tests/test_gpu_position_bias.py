"""The relative position bias and its gradient on the GPU against the float64
definitions, through the binding."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2207_10731_amd import pss
from rows_common import U, numpy64, rounded, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# B, H, Q, K, buckets, distance, both, q_start, starts per sequence
CASES = [
    (1, 1, 1, 1, 8, 64, True, 0, False), (2, 3, 1, 9, 8, 9, False, 8, False),
    (1, 2, 9, 1, 8, 64, True, 0, False), (3, 5, 1, 700, 32, 128, False, 0, True),
    (2, 3, 7, 7, 32, 128, True, 0, False), (2, 4, 33, 65, 32, 128, False, 32, False),
    (1, 3, 64, 64, 16, 30, True, 0, False), (2, 2, 65, 131, 32, 128, True, 0, True),
    (1, 2, 130, 517, 64, 250, False, 387, False), (1, 1, 257, 2050, 32, 128, True, 100, False),
    (2, 1, 20, 4500, 256, 2000, True, 4480, False), (4, 16, 3, 300, 32, 128, False, 297, True),
    (1, 2, 300, 300, 2, 2, False, 0, False), (1, 2, 70, 300, 4, 2, True, 2**29, False),
    (40, 3, 5, 6, 32, 128, True, 0, True), (1, 2, 700, 40, 32, 100, False, 0, False),
]


def _setup(case, seed, starts="some"):
    B, H, Q, K, num, far, both, start, per = case
    rng = np.random.default_rng(seed)
    m = pss.make_position_buckets(num, far, both)
    starts = rng.integers(0, K, B).astype(np.int32) if per else None
    of = lambda n: ro.bucket(n, num, far, both)  # noqa: E731
    first = start + (starts if per else np.zeros(B, np.int64)).astype(np.int64)
    cache = {}
    for f in first:
        if int(f) not in cache:
            cache[int(f)] = ro.bucket_matrix(int(f), Q, K, of)
    buckets = np.stack([cache[int(f)] for f in first])
    return rng, m, buckets, None if starts is None else torch.from_numpy(starts).cuda()


def _frame(shape, dtype, pad):
    """[B][H][Q][K] in an array of 7s, `pad` elements apart from the next row."""
    B, H, Q, K = shape
    return torch.full((B, H, Q, K + pad), 7.0, dtype=dtype, device="cuda")[..., :K]


@pytest.mark.parametrize("dtype,tdtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, dtype, tdtype):
    B, H, Q, K, num = case[:5]
    rng, m, buckets, starts = _setup(case, sum(case[:4]))
    table = torch.from_numpy(rng.normal(0, 1, (num, H))).to("cuda", tdtype)
    for pad, with_scores in ((0, True), (3, True), (0, False), (5, False)):
        scores = None
        if with_scores:
            scores = torch.from_numpy(rng.normal(0, 2, (B, H, Q, K + pad))).to("cuda", dtype)[..., :K]
        out = _frame((B, H, Q, K), dtype, pad)
        pss.pss_position_bias_forward(table, m, out, scores=scores, q_start=case[7], q_starts=starts)
        ref = ro.position_bias(numpy64(table), buckets, numpy64(scores))
        within(out, ref, rounded(ref, U * np.abs(ref), dtype), (pad, with_scores))
        assert pad == 0 or bool((out._base[..., K:] == 7).all())


def test_forward_masked_scores():
    """Masked places: -inf and NaN stay, the type's lowest value stays finite or
    overflows as the float32 sum does; an empty row stays empty."""
    case = (1, 2, 40, 90, 32, 128, True, 0, False)
    rng, m, buckets, _ = _setup(case, 1)
    for dtype in (F32, BF16):
        table = torch.from_numpy(rng.normal(0, 1, (32, 2))).to("cuda", dtype)
        x = torch.from_numpy(rng.normal(0, 2, (1, 2, 40, 90))).to("cuda", dtype)
        x[0, 0, 3] = -float("inf")
        x[0, 1, 5, 40:] = float("nan")
        x[0, 1, 6] = torch.finfo(dtype).min
        out = torch.empty_like(x)
        pss.pss_position_bias_forward(table, m, out, scores=x)
        ref = ro.position_bias(numpy64(table), buckets, numpy64(x))
        assert bool((out[0, 0, 3] == -float("inf")).all()) and bool(out[0, 1, 5, 40:].isnan().all())
        assert bool((out[0, 1, 6] == torch.finfo(dtype).min).all())
        within(out, ref, rounded(ref, U * np.abs(ref), dtype), dtype)


def test_forward_in_place_and_layouts():
    """Scores updated in place; [B][Q][H][K] arrays seen as [B][H][Q][K]; a
    broadcast input (one score row for every head)."""
    case = (3, 4, 21, 50, 32, 128, True, 7, True)
    rng, m, buckets, starts = _setup(case, 2)
    table = torch.from_numpy(rng.normal(0, 1, (32, 4))).to("cuda", F32)
    x = torch.from_numpy(rng.normal(0, 2, (3, 21, 4, 50))).to("cuda", F32).permute(0, 2, 1, 3)
    ref = ro.position_bias(numpy64(table), buckets, numpy64(x))
    out = torch.empty(3, 21, 4, 50, device="cuda").permute(0, 2, 1, 3)
    pss.pss_position_bias_forward(table, m, out, scores=x, q_start=7, q_starts=starts)
    within(out, ref, rounded(ref, U * np.abs(ref), F32), "permuted")
    pss.pss_position_bias_forward(table, m, x, scores=x, q_start=7, q_starts=starts)
    assert torch.equal(x, out)
    one = x[:, :1].expand(3, 4, 21, 50)
    ref = ro.position_bias(numpy64(table), buckets, numpy64(one))
    pss.pss_position_bias_forward(table, m, out, scores=one, q_start=7, q_starts=starts)
    within(out, ref, rounded(ref, U * np.abs(ref), F32), "broadcast")
    g = torch.empty(32, 4, device="cuda")
    pss.pss_position_bias_backward(one, m, g, q_start=7, q_starts=starts)
    a = numpy64(one)
    within(g, ro.position_bias_grad(a, buckets, 32),
           CHAIN * U * ro.position_bias_grad(np.abs(a), buckets, 32), "broadcast gradient")


def test_starts_are_clamped():
    """Whatever the start positions hold, the call stays in its arrays: below 0
    counts as 0, beyond 2^29 as 2^29."""
    m = pss.make_position_buckets(8, 64, True)
    table = torch.arange(8.0, device="cuda")[:, None].contiguous()
    wild = torch.tensor([-5, -2**31, 2**31 - 1, 2**29 + 3], dtype=torch.int32, device="cuda")
    tame = torch.tensor([0, 0, 2**29, 2**29], dtype=torch.int32, device="cuda")
    a, b = (torch.empty(4, 1, 9, 30, device="cuda") for _ in range(2))
    g, h = (torch.empty(8, 1, device="cuda") for _ in range(2))
    x = torch.randn(4, 1, 9, 30, device="cuda")
    for start, out, grad in ((wild, a, g), (tame, b, h)):
        pss.pss_position_bias_forward(table, m, out, q_start=3, q_starts=start)
        pss.pss_position_bias_backward(x, m, grad, q_start=3, q_starts=start)
    assert torch.equal(a, b) and torch.equal(g, h)


# Additions on the longest path of one entry: rows of a tile (at most 512),
# its diagonals and the tiles of one head, each summed by at least 64 lanes and
# a tree: below 1024 for the sizes here.
CHAIN = 1024


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", CASES + [(2, 2, 1000, 1500, 32, 128, False, 500, False),
                                          (300, 2, 1, 100, 32, 128, False, 0, True),
                                          (1, 3, 64, 9000, 64, 5000, True, 3000, False)])
def test_gradient(case, dtype):
    B, H, Q, K, num = case[:5]
    rng, m, buckets, starts = _setup(case, sum(case[:4]))
    for pad in (0, 3):
        g = torch.from_numpy(rng.normal(0.1, 1, (B, H, Q, K + pad))).to("cuda", dtype)[..., :K]
        out = torch.full((num, H), 7.0, device="cuda")
        pss.pss_position_bias_backward(g, m, out, q_start=case[7], q_starts=starts)
        ref = ro.position_bias_grad(numpy64(g), buckets, num)
        mag = ro.position_bias_grad(np.abs(numpy64(g)), buckets, num)
        within(out, ref, CHAIN * U * mag, pad)
        again = torch.empty_like(out)
        pss.pss_position_bias_backward(g, m, again, q_start=case[7], q_starts=starts)
        assert torch.equal(out, again)


def test_gradient_of_own_borders():
    """Repeated borders: buckets that hold no distance get 0; keys ahead fall
    into the bucket of distance 0 on a single side."""
    m = pss.pss_position_buckets(5, 0)
    m.borders[:5] = [0, 0, 3, 3, 9]
    of = lambda n: int(pss.pss_position_buckets_host(m, [n])[0])  # noqa: E731
    buckets = ro.bucket_matrix(10, 30, 50, of)[None]
    g = torch.randn(1, 2, 30, 50, device="cuda")
    out = torch.full((5, 2), 7.0, device="cuda")
    pss.pss_position_bias_backward(g, m, out, q_start=10)
    ref = ro.position_bias_grad(numpy64(g), buckets, 5)
    within(out, ref, CHAIN * U * ro.position_bias_grad(np.abs(numpy64(g)), buckets, 5), "own")
    assert bool((out[0] == 0).all()) and bool((out[2] == 0).all())
    one = pss.pss_position_buckets(1, 0)
    out = torch.empty(1, 2, device="cuda")
    pss.pss_position_bias_backward(g, one, out)
    within(out, numpy64(g).sum((0, 2, 3))[None], CHAIN * U * np.abs(numpy64(g)).sum((0, 2, 3)), "one")


def test_empty_sizes():
    m = pss.make_position_buckets(8, 64, True)
    for shape in ((0, 2, 3, 4), (2, 2, 0, 4), (2, 2, 3, 0)):
        x = torch.empty(shape, device="cuda")
        g = torch.full((8, 2), 7.0, device="cuda")
        pss.pss_position_bias_backward(x, m, g)
        assert bool((g == 0).all())
        pss.pss_position_bias_forward(g, m, x, scores=x)
    x = torch.empty(2, 0, 3, 4, device="cuda")
    pss.pss_position_bias_backward(x, m, torch.empty(8, 0, device="cuda"))


def test_rows_beyond_32_bits():
    """Query rows that begin past 2^32 elements."""
    stride, K = 2**31 + 40, 200
    base = torch.empty(2 * stride + K, dtype=BF16, device="cuda")
    x = base.as_strided((1, 1, 3, K), (3 * stride, 3 * stride, stride, 1))
    case = (1, 1, 3, K, 32, 128, True, 60, False)
    rng, m, buckets, _ = _setup(case, 3)
    x.copy_(torch.from_numpy(rng.normal(0, 1, (1, 1, 3, K))))
    table = torch.from_numpy(rng.normal(0, 1, (32, 1))).to("cuda", F32)
    g = torch.empty(32, 1, device="cuda")
    pss.pss_position_bias_backward(x, m, g, q_start=60)
    a = numpy64(x)
    within(g, ro.position_bias_grad(a, buckets, 32),
           CHAIN * U * ro.position_bias_grad(np.abs(a), buckets, 32), "gradient")
    ref = ro.position_bias(numpy64(table), buckets, a)
    pss.pss_position_bias_forward(table, m, x, scores=x, q_start=60)
    within(x, ref, rounded(ref, U * np.abs(ref), BF16), "forward")


def test_captured_calls_and_streams():
    """Two captured gradient calls replayed in turn with eager ones between, and
    calls on two streams: the same bits as alone."""
    rng, m, _, _ = _setup((1, 1, 1, 1, 32, 128, True, 0, False), 4)
    xs = [torch.randn(2, 3, 200, 300, device="cuda"), torch.randn(4, 3, 50, 900, device="cuda")]
    want = []
    for x in xs:
        g = torch.empty(32, 3, device="cuda")
        pss.pss_position_bias_backward(x, m, g)
        want.append(g)
    outs = [torch.empty(32, 3, device="cuda") for _ in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for x, o in zip(xs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            pss.pss_position_bias_backward(x, m, o)
        graphs.append(graph)
    eager = torch.empty(32, 3, device="cuda")
    for k in range(4):
        for i in (0, 1):
            outs[i].fill_(7.0)
            graphs[i].replay()
            pss.pss_position_bias_backward(xs[1 - i], m, eager)
            assert torch.equal(eager, want[1 - i])
            assert torch.equal(outs[i], want[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for st, x, o in zip(streams, xs, outs):
            pss.pss_position_bias_backward(x, m, o, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_binding_refuses():
    m = pss.make_position_buckets(8, 64, True)
    x = torch.zeros(2, 3, 4, 5, device="cuda")
    t = torch.zeros(8, 3, device="cuda")
    ok = torch.zeros(2, dtype=torch.int32, device="cuda")
    for table in (t[:7], t[:, :2], t.half(), t.cpu(), torch.zeros(3, 8, device="cuda").t()):
        with pytest.raises((ValueError, TypeError)):
            pss.pss_position_bias_forward(table, m, x)
        with pytest.raises((ValueError, TypeError)):
            pss.pss_position_bias_backward(x, m, table)
    for scores in (x[:1], x.bfloat16(), x.cpu(), torch.zeros(2, 3, 5, 4, device="cuda").mT, x[0]):
        with pytest.raises((ValueError, TypeError)):
            pss.pss_position_bias_forward(t, m, x, scores=scores)
    for starts in (ok[:1], ok.long(), ok.cpu()):
        with pytest.raises((ValueError, TypeError)):
            pss.pss_position_bias_forward(t, m, x, q_starts=starts)
        with pytest.raises((ValueError, TypeError)):
            pss.pss_position_bias_backward(x, m, t, q_starts=starts)
    with pytest.raises(pss.PssError):
        pss.pss_position_bias_forward(t, m, x, q_start=-1)
    with pytest.raises(pss.PssError):  # an output that overlaps itself
        pss.pss_position_bias_forward(t, m, x[:1].expand(2, 3, 4, 5))
