"""Evictions whose sizes are given as far more than there is."""
import ctypes as C

import pytest

from tests.test_paged_evict_rows_gpu import DEV, free_pages
from tests.test_paged_gpu import Case
from tests.test_paged_weigh_gpu import evict

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_length", [2 ** 31 - 1, 2 ** 31 - 9])
@pytest.mark.parametrize("lengths,keep,heads", [([90], [12], 1), ([9000, 20], [800, 5], 1), ([300] * 40, [100] * 40, 4)])
def test_any_max_length_sizes_an_eviction(max_length, lengths, keep, heads):
    evict(lengths, keep, heads, n_sink=2, max_length=max_length)


def test_room_for_any_number_of_positions():
    """kept_len near 2^31 (the row is as long as what stays; nothing is written behind it)."""
    c = Case([60], [0], 1, 1, 64, spare=2).fill()
    free = free_pages(c)
    to, keep, kept = torch.tensor([free], **DEV), torch.tensor([20], **DEV), torch.full((32,), -9, **DEV)
    w = torch.rand(c.kv.n_pages, 1, 16, device="cuda")
    for length in (2 ** 31 - 1, 2 ** 31 - 100):
        kept.fill_(-9)
        batch = c.batch()
        c.kv._check(c.kv.lib.scalekv_paged_evict(c.kv.handle, c.layer, C.byref(batch.struct), to.data_ptr(), 2, 2, keep.data_ptr(), w.data_ptr(), 3, 17, kept.data_ptr(), 2 ** 31 - 1, length,
                                                 torch.cuda.current_stream().cuda_stream))
        c.kv.scalekv_paged_sync()
        assert kept.tolist() == [0, 1, 2, *range(43, 60)] + [-9] * 12
        assert torch.equal(w[free[1], 0, :4], w[c.table[0, 3].item(), 0, 8:12])
