"""Sizes that the paged cache accepts beyond the usual ones: pages longer than a key tile, more sequences than a launch deals out, more sequences and heads
than it counts parts of; against fp64."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from tests import stream_rule as sr
from tests.test_paged_dealt_parts_gpu import check
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 128), ("q8", 64), ("bf16", 64)])
@pytest.mark.parametrize("page", [256, 512, 4096])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [40, 1, 130, 0], [200, 300, 257, 5]])
def test_pages_longer_than_a_key_tile(page, new, store, d):
    lengths = [700, 1100, 257, 5]
    c = Case(lengths, new, 2, 3, d, store, page=page).fill()
    K, V = c.kv.scalekv_paged_read(c.layer, c.batch(lengths), dtype=torch.float32)
    for got, x in ((K, c.K), (V, c.V)):
        assert np.array_equal(got.cpu().numpy(), po.stored(x, store))
    check(c, max(lengths))
    check(c, max(lengths), window=300, n_sink=20)


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("n,heads", [(600, 1), (600, 8), (513, 3)])
def test_more_sequences_than_are_dealt_out_or_counted(n, heads, store):
    lengths = [int(x) for x in np.random.default_rng(n).integers(0, 120, n)]
    c = Case([max(length, 1) for length in lengths], [0 if b % 11 == 3 else 1 for b in range(n)], heads, 2, 128, store).fill()
    assert sr.cut(sr.slots(128, store, 2), n, n * heads, sum(c.new) * heads * 2, 1 << 20)[1] == 0
    check(c, 1 << 20)
    # chunks beside them
    counts = [min(40, length) if b % 50 == 7 else (0 if b % 11 == 3 else 1) for b, length in enumerate(c.lengths)]
    c.new, c.Q = counts, po.to_bf16(c.rng.standard_normal((sum(counts), heads * 2, 128)).astype(np.float32))
    check(c, max(c.lengths))
