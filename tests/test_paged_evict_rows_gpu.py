"""Rows of positions, and of pages to move to, that overlap."""
import pytest

from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = dict(dtype=torch.int32, device="cuda")


def free_pages(c):
    used = set(c.table.cpu().numpy().ravel().tolist())
    return [p for p in range(c.kv.n_pages) if p not in used]


@pytest.mark.parametrize("which", ["kept", "kept of a head", "to_table"])
def test_rows_that_overlap_are_refused(which):
    """Positions, and pages to move to, are every row's own: one that begins inside another would be written by both."""
    c = Case([60, 50], [0, 0], 2, 1, 64, spare=4).fill()
    free = free_pages(c)
    to, keep = torch.tensor([free[:2], free[2:4]], **DEV), torch.tensor([16, 16], **DEV)
    kept = torch.zeros(2, 2, 16, **DEV)
    if which == "kept":
        kept = torch.zeros(1, 1, 16, **DEV).expand(2, 2, 16)
    elif which == "kept of a head":
        kept = torch.zeros(200, **DEV).as_strided((2, 2, 16), (16, 8, 1))
    else:
        to = to[:1].expand(2, 2)
    w = torch.rand(c.kv.n_pages, 2, 16, device="cuda")
    old, pool = w.clone(), c.kv.pool.clone()
    with pytest.raises(binding.ScaleKVError, match="overlap"):
        c.kv.scalekv_paged_evict(c.layer, c.batch(), to, keep, w, kept=kept)
    c.kv.scalekv_paged_sync()
    assert torch.equal(w, old) and torch.equal(c.kv.pool, pool) and not kept.any()


def test_one_row_overlaps_with_none():
    c = Case([60], [0], 1, 1, 64, spare=1).fill()
    kept = torch.zeros(1, 1, 16, **DEV).as_strided((1, 1, 16), (3, 3, 1))
    w = torch.rand(c.kv.n_pages, 1, 16, device="cuda")
    c.kv.scalekv_paged_evict(c.layer, c.batch(), torch.tensor([free_pages(c)], **DEV), torch.tensor([16], **DEV), w, n_recent=16, kept=kept)
    c.kv.scalekv_paged_sync()
    assert kept[0, 0].tolist() == list(range(44, 60))
