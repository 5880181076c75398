"""The bias table's gradient where every sum is exact, so that an element lost or
taken twice shows however many a bucket holds; and the bias of few queries under
maps whose borders lie beyond the list of distances."""
import numpy as np
import pytest
import torch

from paper_2207_10731_amd import pss
from rows_common import numpy64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _map(borders, both):
    side = len(borders)
    m = pss.pss_position_buckets(side * (1 + both), int(both))
    m.borders[:side] = borders
    return m


def _buckets(m, first, Q, K):
    """[Q][K] from the definition: the last border at or below the distance."""
    both = bool(m.bidirectional)
    side = m.num_buckets // (1 + both)
    n = (first + np.arange(Q))[:, None] - np.arange(K)[None, :]
    far = np.abs(n) if both else np.maximum(n, 0)
    j = np.searchsorted(np.array(m.borders[:side]), far, side="right") - 1
    return j + side * (n < 0) * both


def _exact(m, B, H, Q, K, dtype, start, per, pad, seed):
    """Gradients 1, 2 and 3: every partial sum of a bucket is a whole number below
    2^24, so that float32 sums are exact in any order."""
    assert B * Q * K * 3 < 2**24
    rng = np.random.default_rng(seed)
    g = rng.integers(1, 4, (B, H, Q, K + pad)).astype(np.float32)
    starts = rng.integers(0, K, B).astype(np.int32) if per else None
    x = torch.from_numpy(g).to("cuda", dtype)[..., :K]
    out = torch.full((m.num_buckets, H), 7.0, device="cuda")
    pss.pss_position_bias_backward(x, m, out, q_start=start,
                                   q_starts=None if starts is None else torch.from_numpy(starts).cuda())
    want = np.zeros((m.num_buckets, H))
    for b in range(B):
        at = _buckets(m, start + (int(starts[b]) if per else 0), Q, K).reshape(-1)
        for h in range(H):
            want[:, h] += np.bincount(at, g[b, h, :, :K].reshape(-1), m.num_buckets)
    assert np.array_equal(numpy64(out), want), np.argwhere(numpy64(out) != want)[:5].tolist()


# B, H, Q, K, q_start, starts per sequence: one block and many, several units to a
# wavefront, groups of 8 to 64 lanes, steps of 1, 2, 4 and 8 queries, rows that end
# inside a vector
SIZES = [
    (1, 1, 1, 1, 0, False), (1, 2, 1, 700, 350, False), (2, 3, 2, 9, 4, False), (64, 4, 1, 4099, 0, True),
    (33, 3, 2, 3001, 5, True), (17, 2, 4, 2051, 0, True), (9, 2, 3, 4096, 100, True),
    (300, 5, 1, 100, 0, True), (700, 3, 20, 20, 0, False), (2, 2, 1000, 1500, 500, False),
    (3, 2, 700, 1303, 0, True), (1, 2, 2048, 2048, 0, False), (1, 1, 2047, 2600, 553, False),
    (5, 70, 65, 131, 0, True), (1, 3, 4000, 37, 0, False), (2, 2, 130, 4, 0, False), (40, 2, 7, 5, 0, True),
]
USUAL = [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("case", SIZES)
def test_gradient_counts_every_pair_once(case, both, dtype):
    B, H, Q, K, start, per = case
    m = _map(USUAL, both)
    for pad in (0, 3):
        _exact(m, B, H, Q, K, dtype, start, per, pad, Q + K + pad)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("borders", [[0], [0, 0, 3, 3, 9], [0, 1024], [0, 1, 511, 1000, 1024], [0, 1025],
                                     [0, 5, 300, 2000, 2001], [0, 2**31 - 1]])
def test_gradient_of_borders_near_and_far(borders, both, dtype):
    """The last border at either side of the window's limit, one bucket, repeated
    borders."""
    m = _map(borders, both)
    for B, H, Q, K, start, per in ((2, 2, 300, 1503, 700, False), (20, 2, 1, 4096, 0, True),
                                   (1, 2, 1, 2400, 2399, False), (3, 2, 9, 2300, 1200, True)):
        _exact(m, B, H, Q, K, dtype, start, per, 0, K)


# Borders beyond 1024: keys are searched for.  Runs of borders one or two apart cross
# several inside a vector, long gaps leave vectors in one bucket.
FAR = [[0, 1, 2, 3, 5, 6, 900, 901, 903, 2000, 2001, 2002, 2003, 2500], [0, 1500], [0, 0, 7, 7, 7, 1100, 1100],
       [0, 1, 1025], list(range(0, 1280, 10))]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("borders", FAR)
@pytest.mark.parametrize("Q,K,start", [(1, 6001, 3000), (3, 5000, 2490), (7, 4099, 1030), (2, 37, 1100),
                                       (1, 5000, 0), (5, 2600, 2595)])
def test_few_queries_of_far_borders(Q, K, start, borders, both, dtype):
    """The bias alone, of a table of bfloat16 numbers: exact."""
    m = _map(borders, both)
    rng = np.random.default_rng(K)
    B, H = 3, 2
    table = torch.from_numpy(rng.normal(0, 1, (m.num_buckets, H))).to("cuda", BF16)
    starts = np.array([0, 1, 611], np.int32)
    out = torch.full((B, H, Q, K + 5), 7.0, dtype=dtype, device="cuda")
    pss.pss_position_bias_forward(table, m, out[..., :K], q_start=start,
                                  q_starts=torch.from_numpy(starts).cuda())
    t = numpy64(table)
    want = np.stack([np.moveaxis(t[_buckets(m, start + int(s), Q, K)], -1, 0) for s in starts])
    assert np.array_equal(numpy64(out[..., :K]), want)
    assert bool((out[..., K:] == 7.0).all())
    # added to scores in place, the same sum as of the bias alone
    x = torch.from_numpy(rng.normal(0, 2, (B, H, Q, K))).to("cuda", dtype)
    both_sum = (x.float() + out[..., :K].float()).to(dtype)
    pss.pss_position_bias_forward(table, m, x, scores=x, q_start=start,
                                  q_starts=torch.from_numpy(starts).cuda())
    assert torch.equal(x, both_sum)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 7, 8, 9, 15])
def test_gradient_of_rows_of_few_keys(K, dtype):
    """Rows shorter than a vector, of one and just above, near and far borders."""
    for borders, both in ((USUAL, True), ([0, 3, 2000], True), ([0, 1, 5, 1100], False)):
        for B, H, Q, start, per in ((3, 2, 70, 0, True), (1, 3, 1, 1102, False), (50, 1, 9, 1095, False)):
            _exact(_map(borders, both), B, H, Q, K, dtype, start, per, 0, K)
