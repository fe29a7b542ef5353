"""The paged cache's own memory on streams other than the one it was made on."""
import gc

import pytest

from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
COUNTERS = 256 + 4096 * 4                  # the status word and the counts of parts, which begin at zero
LONG = 400_000_000                         # cycles: a fifth of a second


def test_a_handle_made_while_its_memory_is_still_written():
    """The allocator gives a stream memory whose last user on that stream has not run yet; what the handle sets to zero must stay zero."""
    size = binding.PagedKV(1, 4, 1, 64).workspace_bytes
    pool = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = torch.empty(size, dtype=torch.uint8, device="cuda")
        at = x.data_ptr()
        torch.cuda._sleep(LONG)
        x.fill_(255)
        del x
        kv = binding.PagedKV(1, 4, 1, 64, pool=pool)
    assert kv.workspace.data_ptr() == at
    torch.cuda.synchronize()
    assert not bool(kv.workspace[:COUNTERS].any())
    kv.scalekv_paged_sync()


def test_a_handle_that_goes_while_another_stream_still_works_for_it():
    """Its memory is the allocator's again, but not anybody else's before that stream is through."""
    c = Case([300, 200], [1, 1], 1, 2, 64).fill()
    Q, batch = torch.from_numpy(c.Q).cuda().bfloat16(), c.batch()
    O = torch.empty_like(Q)
    want = c.kv.scalekv_paged_attend(c.layer, batch, Q).clone()
    sizes, at = (c.kv.workspace_bytes, c.kv.pool.numel()), (c.kv.workspace.data_ptr(), c.kv.pool.data_ptr())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
        c.kv.scalekv_paged_attend(c.layer, batch, Q, O)
    c.kv = None
    gc.collect()
    others = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
    assert not side.query()                                       # (or nothing has been shown)
    assert not {x.data_ptr() for x in others} & set(at)
    torch.cuda.synchronize()
    assert torch.equal(O, want)
