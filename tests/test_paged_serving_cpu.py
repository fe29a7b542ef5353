"""The page book of drafts and evictions, and what drafted tokens see of one another, on the host."""
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import pipeline


def test_drafts_are_taken_back():
    s = pipeline.Sequences(10, 16, 2, 100)
    s.extend([30, 5])
    s.extend([20, 0])
    held = [row[:] for row in s.table]
    s.retract([17, 0])                                                      # 33 entries: still three pages
    assert s.lengths == [33, 5] and s.table[0][:3] == held[0][:3] and s.table[0][3] == -1 and len(s.free) == 6
    s.retract([1, 5])
    assert s.lengths == [32, 0] and s.table[1][0] == -1 and len(s.free) == 8 and sorted(s.free + s.table[0][:2]) == list(range(10))
    for wrong in ([33, 0], [0, 1], [-1, 0], [0]):
        with pytest.raises(ValueError):
            s.retract(wrong)
    assert s.lengths == [32, 0] and len(s.free) == 8


def test_survivors_move_to_free_pages():
    s = pipeline.Sequences(12, 16, 3, 100)
    s.extend([80, 20, 3])                                                   # 5 + 2 + 1 pages
    with pytest.raises(MemoryError):
        s.survivors([80, 20, 3])
    with pytest.raises(ValueError):
        s.survivors([1, 2, -3])
    old = [row[:] for row in s.table]
    table = s.survivors([17, 16, 100])
    assert [sum(p >= 0 for p in row) for row in table] == [2, 1, 1] and s.table == old and len(s.free) == 4
    assert not {p for row in table for p in row if p >= 0} & {p for row in old for p in row if p >= 0}
    s.survive(table, [17, 16, 100])
    assert s.lengths == [17, 16, 3] and s.table == table and sorted(s.free + [p for row in table for p in row if p >= 0]) == list(range(12))
    s.extend([15, 1, 0])
    assert s.lengths == [32, 17, 3] and len(s.free) == 7
    s.trim(window=10)
    with pytest.raises(ValueError, match="window"):
        s.survivors([1, 1, 1])


def test_trees():
    parents = [[-1, 0, 0, 2, -1], [], [-1] + list(range(39))]
    bits, depths = pipeline.tree_bits(parents)
    sees = [[[0], [0, 1], [0, 2], [0, 2, 3], [4]], [], [list(range(i + 1)) for i in range(40)]]
    assert [row for s in sees for row in po.draft_bits(s, 2).tolist()] == bits
    assert depths == [0, 1, 1, 2, 0] + list(range(40))
    assert pipeline.tree_bits([[], []]) == ([], [])
    for wrong in ([0], [-1, 1], [-1, -2], [-1, 2, 0]):
        with pytest.raises(ValueError):
            pipeline.tree_bits([wrong])
