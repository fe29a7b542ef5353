"""Drafts of which more would be accepted than a path names, or than were drafted."""
import pytest

from tests.test_paged_evict_no_room_gpu import told
from tests.test_paged_evict_rows_gpu import DEV
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_accepted_tokens_that_no_path_names_are_told():
    c = Case([20, 9], [8, 4], 2, 1, 64).fill()
    pool = c.kv.pool.clone()
    none = torch.zeros(2, 0, **DEV)
    c.kv.scalekv_paged_accept(c.batch(), none, torch.tensor([0, 0], **DEV))
    c.kv.scalekv_paged_sync()
    for counts in ([0, 1], [-1, 0]):
        c.kv.scalekv_paged_accept(c.batch(), none, torch.tensor(counts, **DEV))
        told(c)
    path = torch.zeros(2, 3, **DEV)
    nobody = c.batch(new=[0, 0])                                      # a step without a draft
    c.kv.scalekv_paged_accept(nobody, path, torch.tensor([0, 0], **DEV))
    c.kv.scalekv_paged_sync()
    c.kv.scalekv_paged_accept(nobody, path, torch.tensor([1, 0], **DEV))
    told(c)
    assert torch.equal(c.kv.pool, pool)
