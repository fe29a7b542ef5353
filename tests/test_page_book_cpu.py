"""The sequences' page book at its edges."""
import pytest

from paper_2505_19602_b200 import pipeline


def book():
    s = pipeline.Sequences(12, 16, 3, 100)
    s.extend([80, 33, 0])
    return s


def state(s):
    return [list(row) for row in s.table], list(s.lengths), sorted(s.free)


def test_no_window_hides_no_page():
    for sinks in (0, 3):
        s = book()
        before = state(s)
        s.trim(0, sinks)
        assert state(s) == before
    s = book()
    s.trim(1)                                      # the next token of sequence 0, at 80, sees itself only; sequence 1's, at 33, lies in the page of entry 32
    assert [p >= 0 for p in s.table[0]] == [False] * 7 and [p >= 0 for p in s.table[1][:3]] == [False, False, True]


@pytest.mark.parametrize("window,n_sink", [(-1, 0), (5, -1)])
def test_windows_that_are_none(window, n_sink):
    s = book()
    before = state(s)
    with pytest.raises(ValueError):
        s.trim(window, n_sink)
    assert state(s) == before


@pytest.mark.parametrize("new", [[1, 1], [1, 1, 1, 1], [], [1, -1, 0]])
def test_tokens_for_every_sequence(new):
    s = book()
    before = state(s)
    with pytest.raises(ValueError):
        s.extend(new)
    assert state(s) == before
