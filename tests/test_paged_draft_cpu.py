"""pipeline.draft_step without a GPU: paths that cannot be, and steps that end early, leave the page book as it was."""
import pytest

from paper_2505_19602_b200 import pipeline

torch = pytest.importorskip("torch")


class Cache:
    """Takes the calls of a PagedKV down."""
    n_layers, device, device_index, store = 2, torch.device("cpu"), 0, "q8"

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if not name.startswith("scalekv_"):
            raise AttributeError(name)

        def call(*args, **kw):
            self.calls.append(name[len("scalekv_paged_"):])
            return torch.zeros(1)

        return call


@pytest.fixture
def book(monkeypatch):
    s = pipeline.Sequences(12, 16, 2, 90)
    s.extend([30, 5])
    monkeypatch.setattr(s, "batch", lambda new, device=0: None)
    return s


def state(s):
    return list(s.lengths), [row[:] for row in s.table], sorted(s.free)


PARENTS = [[-1, 0, 1] + [-1] * 17, [-1, 0, 0]]


def rows(l):
    return torch.zeros(23, 2, 64), None, None


@pytest.mark.parametrize("paths", [[[0, 1], [2, 1]], [[0, 0], []], [[-1], []], [[20], []], [[], [3]], [[0]], [[0], [0], [0]], [list(range(21)), []], []])
def test_a_path_that_cannot_be_is_refused_and_the_draft_taken_back(book, paths):
    kv, before = Cache(), state(book)
    with pytest.raises(ValueError, match="path"):
        pipeline.draft_step(kv, book, PARENTS, rows, lambda out: paths)
    assert state(book) == before and "accept" not in kv.calls


@pytest.mark.parametrize("where", ["rows", "accept"])
def test_a_step_that_ends_early_takes_the_draft_back(book, where):
    def fail(x):
        raise KeyError(where)

    kv, before = Cache(), state(book)
    with pytest.raises(KeyError, match=where):
        pipeline.draft_step(kv, book, PARENTS, fail if where == "rows" else rows, fail if where == "accept" else lambda out: [[], []])
    assert state(book) == before and "accept" not in kv.calls


def test_a_draft_that_stays(book):
    kv = Cache()
    out, paths = pipeline.draft_step(kv, book, PARENTS, rows, lambda out: [[0, 1, 2], []])
    assert paths == [[0, 1, 2], []] and len(out) == 2 and book.lengths == [33, 5]
    assert kv.calls == ["write", "attend_tree"] * 2 + ["accept"]
