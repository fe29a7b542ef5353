"""Evictions that have no room for what would stay."""
import pytest

from paper_2505_19602_b200 import binding
from tests.test_paged_evict_rows_gpu import DEV
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def told(c):
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()
    c.kv.workspace[:4].zero_()


@pytest.mark.parametrize("given", [True, False])
def test_an_eviction_without_room_is_told(given):
    c = Case([60, 0], [0, 0], 2, 1, 64, spare=2).fill()
    w = torch.rand(c.kv.n_pages, 2, 16, device="cuda")
    old, pool = w.clone(), c.kv.pool.clone()
    to = torch.zeros(2, 0, **DEV)
    kept = torch.zeros(2, 2, 0, **DEV) if given else None
    c.kv.scalekv_paged_evict(c.layer, c.batch(), to, torch.tensor([0, 9], **DEV), w, kept=kept)      # nothing would stay
    c.kv.scalekv_paged_sync()
    c.kv.scalekv_paged_evict(c.layer, c.batch(), to, torch.tensor([1, 9], **DEV), w, kept=kept)
    told(c)
    c.kv.scalekv_paged_evict(c.layer, c.batch(), to, torch.tensor([0, -1], **DEV), w, kept=kept)
    told(c)
    assert torch.equal(w, old) and torch.equal(c.kv.pool, pool)
