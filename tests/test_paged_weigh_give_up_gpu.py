"""Sums that nothing may change: of entries beside holes in a table, and of all once a device-side wait has given up."""
import pytest

from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case
from tests.test_paged_weigh_infinite_gpu import queries, sums

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TIMEOUT = binding.STATUS_NAMES.index("TIMEOUT")


@pytest.mark.parametrize("new", [1, 60])
def test_holes_behind_a_window_change_no_sum(new):
    c = Case([400], [new], 1, 1, 64, page=16).fill()
    lo = (400 - new - 50 + 1) // 16
    lse, old, got = torch.full((new, 1), 4.0, device="cuda"), sums(c), []
    pages = c.table[0].clone()
    for hole in (None, -3):
        if hole is not None:
            c.table[0, 1:lo] = hole
        w = old.clone()
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, w, window=50, n_sink=3, decay=0.5)
        c.kv.scalekv_paged_sync()
        got.append(w)
    assert torch.equal(*got) and torch.equal(got[0][pages[1:lo].long()], old[pages[1:lo].long()]) and not torch.equal(got[0], old)


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("lengths,new", [([3001, 70], [40, 0]), ([200], [150])])
def test_no_sum_is_stored_once_a_wait_gave_up(store, lengths, new):
    """(the status word is set from the host; no wait runs out here)"""
    c = Case(lengths, new, 1, 2, 128, store, page=64).fill()
    lse, old = torch.full((sum(new), 2), 3.0, device="cuda"), sums(c)
    want = old.clone()
    c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, want, decay=0.5)
    c.kv.scalekv_paged_sync()
    c.kv.workspace[:4].view(torch.int32).fill_(TIMEOUT)
    w = old.clone()
    c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, w, decay=0.5)
    with pytest.raises(binding.ScaleKVError, match="TIMEOUT"):
        c.kv.scalekv_paged_sync()
    assert torch.equal(w, old)
    c.kv.workspace[:4].zero_()
    c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, w, decay=0.5)
    c.kv.scalekv_paged_sync()
    assert torch.equal(w, want) and not torch.equal(w, old)
