"""The paged cache once a device-side wait has given up (the status word is set from the host; no wait runs out here): what chunks left before is not
taken for results."""
import pytest

from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TIMEOUT = binding.STATUS_NAMES.index("TIMEOUT")


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("lengths,new", [([3001], [40]),          # every item is shared by CTAs and joined by a launch behind them
                                         ([200], [150])])         # items of their own
def test_no_row_is_stored(store, lengths, new):
    c = Case(lengths, new, 1, 2, 128, store, page=64).fill()
    launches = c.kv.scalekv_paged_launch_count()
    c.check()                                                     # (leaves parts in the workspace)
    assert c.kv.scalekv_paged_launch_count() - launches == (2 if lengths == [3001] else 1)
    c.kv.workspace[:4].view(torch.int32).fill_(TIMEOUT)
    Q = torch.from_numpy(c.Q).cuda().bfloat16()
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device="cuda")
    c.kv.scalekv_paged_attend(c.layer, c.batch(), Q, O, lse)
    with pytest.raises(binding.ScaleKVError, match="TIMEOUT"):
        c.kv.scalekv_paged_sync()
    assert bool((O == 7).all()) and bool((lse == 7).all())
    c.kv.workspace[:4].zero_()
    c.check()
