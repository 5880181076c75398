"""The position of the first query as the binding hands it on: the value at the
call, whatever integer holds it, and no other type."""
import numpy as np
import pytest
import torch

from paper_2207_10731_amd import pss


class _Library:
    """Stands for the library: keeps the q_start of each call."""

    def __init__(self):
        self.starts = []

    def _take(self, params, *rest):
        self.starts.append(params._obj.q_start)
        return pss.PSS_OK

    pss_position_bias_forward = pss_position_bias_backward = _take


@pytest.fixture
def starts(monkeypatch):
    """The q_starts that the library gets from calls on CPU tensors."""
    lib = _Library()
    monkeypatch.setattr(pss, "load_library", lambda: lib)
    monkeypatch.setattr(pss, "_bias_sizes",
                        lambda name, t: (pss._ROW_DTYPES[t.dtype], t.shape, t.dtype, -1))
    monkeypatch.setattr(pss, "_raw_stream", lambda stream, dev: None)
    return lib.starts


MAP = pss.pss_position_buckets(1, 0)
TABLE, SCORES = torch.zeros(1, 3), torch.zeros(2, 3, 1, 9)


def _forward(q_start):
    pss.pss_position_bias_forward(TABLE, MAP, SCORES, scores=SCORES, q_start=q_start)


def _backward(q_start):
    pss.pss_position_bias_backward(SCORES, MAP, TABLE, q_start=q_start)


@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("kind", [torch.tensor, np.array])
def test_a_counter_advanced_in_place(call, kind, starts):
    pos = kind(5)
    for _ in range(3):
        call(pos)
        pos += 1
    assert starts == [5, 6, 7]


@pytest.mark.parametrize("call", [_forward, _backward])
def test_integers_of_every_type(call, starts):
    for v in (6, np.int32(7), np.int64(8), torch.tensor(9, dtype=torch.int32), torch.tensor([10])):
        call(v)
    assert starts == [6, 7, 8, 9, 10]


@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("bad", [9.0, np.float32(9), torch.tensor(9.0), "9", None])
def test_no_other_type_whatever_was_asked_for_before(call, bad, starts):
    with pytest.raises(TypeError):
        call(bad)
    call(9)
    with pytest.raises(TypeError):
        call(bad)
    assert starts == [9]


@pytest.mark.gpu
def test_decode_loop_with_a_counter_in_place():
    """New tokens one after the other: the bias of each is that of its position."""
    m = pss.make_position_buckets(32, 128, False)
    K = 200
    table = torch.randn(32, 3, device="cuda")
    scores = torch.randn(2, 3, 1, K, device="cuda")
    pos = torch.tensor(90)
    out, want = (torch.empty_like(scores) for _ in range(2))
    g, h = (torch.empty(32, 3, device="cuda") for _ in range(2))
    for p in range(90, 96):
        pss.pss_position_bias_forward(table, m, out, scores=scores, q_start=pos)
        pss.pss_position_bias_forward(table, m, want, scores=scores, q_start=p)
        assert torch.equal(out, want)
        pss.pss_position_bias_backward(scores, m, g, q_start=pos)
        pss.pss_position_bias_backward(scores, m, h, q_start=p)
        assert torch.equal(g, h)
        pos += 1


@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("far", [2**64 + 5, 2**64, -2**64 + 7, 2**32, 2**63, -1])
def test_positions_out_of_range_stay_so(call, far, starts):
    """What the library gets is refused there, not a position modulo 2^64."""
    call(far)
    assert not 0 <= starts[0] <= 2**29


@pytest.mark.gpu
def test_positions_out_of_range_are_refused():
    m, x = pss.make_position_buckets(8, 64, True), torch.zeros(2, 3, 4, 5, device="cuda")
    for far in (2**64 + 5, -1, 2**29 + 1):
        with pytest.raises(pss.PssError):
            pss.pss_position_bias_forward(torch.zeros(8, 3, device="cuda"), m, x, q_start=far)
        with pytest.raises(pss.PssError):
            pss.pss_position_bias_backward(x, m, torch.zeros(8, 3, device="cuda"), q_start=far)
