"""Rotated writes, drafts, summed weights and eviction of the paged cache without a GPU: refusals, what is passed on, and the oracle's own rules."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    binding.build_library()
    return binding.load_library()


def test_null_handles(lib):
    rows = binding.scalekv_rows(None, 0, 0)
    assert lib.scalekv_paged_write_rotated(None, 0, None, 1, rows, rows, rows, rows, 0, None, None, 0, None) == 1
    assert lib.scalekv_paged_attend_tree(None, 0, None, 1, rows, rows, None, None, 1, 0.0, None) == 1
    assert lib.scalekv_paged_accept(None, 0, None, None, 0, 0, None, None) == 1
    assert lib.scalekv_paged_weigh(None, 0, None, 1, rows, None, None, 0.0, None, 1.0, None) == 1
    assert lib.scalekv_paged_evict(None, 0, None, None, 0, 0, None, None, 0, 0, None, 0, 0, None) == 1


@pytest.mark.parametrize("wrong", [{"sections": []}, {"sections": [8, 4]}, {"sections": [72]}, {"sections": [16, -8]}, {"sections": [0]},
                                   {"sections": [8], "theta": 0.0}, {"sections": [8], "theta": float("nan")}, {"sections": [1] * 72}])
def test_refused_rotaries(wrong):
    with pytest.raises(ValueError):
        binding.Rotary(**wrong)


def test_rotary_tables():
    r = binding.Rotary([3, 2, 3], theta=100.0)
    assert list(r.struct.axis)[:8] == [0, 0, 0, 1, 1, 2, 2, 2] and (r.n_pairs, r.n_axes, r.struct.adjacent) == (8, 3, 0)
    assert np.allclose(list(r.struct.frequency)[:8], 100.0 ** (-np.arange(8) / 8))
    r = binding.Rotary([3, 2, 3], theta=100.0, own_range=True, in_turn=True, adjacent=True)
    assert list(r.struct.axis)[:8] == [0, 1, 2, 0, 1, 2, 0, 2] and r.struct.adjacent == 1
    assert np.allclose(list(r.struct.frequency)[:8], [1, 1, 1, 100 ** (-1 / 3), 100 ** (-1 / 2), 100 ** (-1 / 3), 100 ** (-2 / 3), 100 ** (-2 / 3)])
    assert binding.Rotary([64]).n_pairs == 64 and binding.Rotary([0, 8]).struct.axis[0] == 1


def test_native_calls_refuse_what_does_not_fit():
    call = binding.load_call()
    x, i = torch.zeros(3, 2, 64), torch.zeros(3, 2, dtype=torch.int32)
    f = torch.zeros(3, 2)
    for act, error, what in [
            (lambda: call.paged_write_rotated(0, 0, 0, 0, 3, 2, 64, 0, x, x, x, x, 0, 1, i, 0), ValueError, "device"),
            (lambda: call.paged_write_rotated(0, 0, 0, 0, 4, 2, 64, 0, x, x, x, x, 0, 1, i, 0), ValueError, "shape"),
            (lambda: call.paged_write_rotated(0, 0), TypeError, "arguments"),
            (lambda: call.paged_attend_tree(0, 0, 0, 0, 3, 64, 0, None, x, None, i, 0.0, 0), TypeError, "Q"),
            (lambda: call.paged_attend_tree(0, 0, 0, 0, 3, 64, 0, x.bfloat16(), x, None, i, 0.0, 0), ValueError, "Q"),
            (lambda: call.paged_accept(0, 0, -1, 0, 3, 0, None, i, 0), TypeError, "path"),
            (lambda: call.paged_accept(0, 0, -1, 0, 3, 0, i, i[:, 0], 0), ValueError, "device"),
            (lambda: call.paged_accept(0, 0, -1, 0, 4, 0, i, i[:, 0], 0), ValueError, "shape"),
            (lambda: call.paged_weigh(0, 0, 0, 0, 3, 64, 0, x, f, x, 3, 2, 64, True, -1, 0, 1.0, 0.0, 0), ValueError, "window"),
            (lambda: call.paged_weigh(0, 0, 0, 0, 3, 64, 0, x, f, x, 3, 2, 64, True, 0, 2 ** 31, 1.0, 0.0, 0), ValueError, "n_sink"),
            (lambda: call.paged_evict(0, 0, 0, 0, 3, 0, i, i[:, 0], x, 3, 2, 64, -1, 0, i, 0), ValueError, "n_sink"),
            (lambda: call.paged_evict(0, 0, 0, 0, 3, 0, i, i[:, 0], x, 3, 2, 64, 0, 2 ** 40, i, 0), ValueError, "n_recent"),
            (lambda: call.paged_evict(0, 0, 0, 0, 3, 0, i.long(), i[:, 0], x, 3, 2, 64, 0, 0, i, 0), ValueError, "to_table")]:
        with pytest.raises(error, match=what):
            act()


def test_oracle_turns():
    x = np.arange(12.0).reshape(1, 1, 12)
    y, A = po.turned(x, np.array([[1], [2]]), [0, 1], [np.pi / 2, np.pi / 4], False)      # a quarter and a half of a half turn
    assert np.allclose(y[0, 0, :4], [-2, -3, 0, 1]) and np.array_equal(y[0, 0, 4:], x[0, 0, 4:]) and A[0, 0, :5].tolist() == [2, 4, 2, 4, 0]
    y, _ = po.turned(x, np.array([[1], [2]]), [0, 1], [np.pi / 2, np.pi / 4], True)
    assert np.allclose(y[0, 0, :4], [-1, 0, -3, 2])


def test_oracle_drafts():
    seen = po.draft_visible([[0], [0, 1], [2]], 5)
    assert seen.astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 0, 0, 1]]
    assert po.draft_visible([[], [1]], 1).astype(int).tolist() == [[0], [1]]                # a draft longer than the cache: its first token is nowhere
    assert po.draft_bits([[0, 31, 32], []], 2).tolist() == [[-2 ** 31 + 1, 1], [0, 0]]


def test_oracle_weights():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((3, 4)), rng.standard_normal((6, 4))
    seen = po.visible(3, 6, True, 0, 0)
    _, lse, _, _ = po.attend(q, k, k, seen, 0.5)
    got, _, _ = po.attention_got(q, k, lse, seen, 0.5)
    assert np.isclose(got.sum(), 3) and got[5] < 1                                          # every row pays one in all
    lse[1] = -np.inf
    assert np.isclose(po.attention_got(q, k, lse, seen, 0.5)[0].sum(), 2)


def test_oracle_eviction():
    w = np.array([5, 1, 3, 3, np.nan, 0, -0.0, 9], np.float32)
    assert po.stays(w, 3, 0, 0).tolist() == [0, 2, 7] and po.stays(w, 3, 1, 1).tolist() == [0, 2, 7]
    assert po.stays(w, 4, 2, 1).tolist() == [0, 1, 2, 7] and po.stays(w, 7, 0, 0).tolist() == [0, 1, 2, 3, 5, 6, 7]
    assert po.stays(w, 6, 0, 0).tolist() == [0, 1, 2, 3, 5, 7] and po.stays(w, 99, 3, 99).tolist() == list(range(8)) and po.stays(w, 0, 3, 3).tolist() == []
    assert po.stays(w, 3, 2, 5).tolist() == [0, 1, 7] and po.stays(w, 2, 5, 5).tolist() == [0, 1]
