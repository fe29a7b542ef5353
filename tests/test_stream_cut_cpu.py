"""How the streaming attention cuts sequences: what the parts of a launch may be, whatever the sizes."""
import random

import pytest

from tests import stream_rule as sr


def test_parts_fit_the_workspace_and_the_counters():
    r = random.Random(1)
    for _ in range(20000):
        d, store, rows_each = r.choice([64, 128]), r.choice(["q8", "bf16"]), r.choice([1, 4, 8, 9, 16, 24, 32])
        n_seqs, heads = r.choice([1, 2, 3, 31, 64, 511, 512, 513, 5000]), r.choice([1, 2, 8, 64, 300])
        tiles = 1 if rows_each <= 16 else 2
        items, rows, keys = n_seqs * heads * tiles, n_seqs * heads * rows_each, int(10 ** r.uniform(0, 8))
        split, most = sr.cut(sr.slots(d, store, rows_each), n_seqs, items, rows, keys)
        assert split >= 1 and (split == 1 or (split * rows <= sr.library().part_rows() and split <= sr.library().most() and items <= sr.library().max_counts()))
        if most:
            assert 3 <= most <= sr.library().most() and most * rows <= sr.library().part_rows() and items <= sr.library().max_counts() and n_seqs > 1


def test_what_is_dealt_out_covers_every_step_once_and_fits():
    """The parts that the deal implies, walked as the CTAs do: no more to a sequence and head than there is room for, none of more than a share."""
    r = random.Random(2)
    shares = 0
    for _ in range(3000):
        n_seqs, heads, ctas, most = r.choice([2, 7, 64, 300]), r.choice([1, 3, 8, 16]), 148 * r.choice([2, 3, 4]), r.choice([3, 5, 37, 256])
        top = r.choice([1, 8, 65, 700, 20000])
        steps = [r.randint(1, top) if r.random() < 0.3 else max(1, top // r.choice([1, 30])) for _ in range(n_seqs)]
        items, total = n_seqs * heads, sum(steps) * heads
        split, share = sr.deal(total, max(steps), items, ctas, most)
        assert 1 <= split <= most
        if not share:
            continue
        shares += 1
        assert share * ctas >= total
        first = 0
        for n in steps:
            for _ in range(heads):
                parts = (first + n - 1) // share - first // share + 1
                assert parts <= most
                first += n
    assert 100 < shares < 2900


@pytest.mark.parametrize("d,store,rows,want", [(128, "q8", 8, 4), (128, "q8", 9, 3), (128, "bf16", 8, 2), (128, "bf16", 32, 2), (64, "q8", 32, 4), (64, "bf16", 8, 4)])
def test_ctas_of_an_sm(d, store, rows, want):
    assert sr.slots(d, store, rows, 1) == want
