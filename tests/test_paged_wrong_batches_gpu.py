"""Batches whose starts, lengths or counts are out of range, each call on a handle of its own: what they would lead to is left out, all else is as
it should be, and the call itself says so."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# lengths, starts, tokens, max_new; the tokens that a sequence owns, for those who follow the order of the sequences
WRONG = {
    "tokens behind the last sequence": ([100, 40, 9], [0, 1, 2, 3], 6, 4, [0, 1, 2]),
    "tokens ahead of the first sequence": ([100, 40, 9], [2, 3, 5, 6], 6, 4, [2, 3, 4, 5]),
    "a first start below zero": ([100, 40, 9], [-1, 1, 2, 6], 6, 4, [1, 2, 3, 4, 5]),
    "a first start behind the second": ([100, 40, 9], [5, 1, 2, 6], 6, 4, [1, 2, 3, 4, 5]),
    "starts that go back, first and last as they should be": ([100, 40, 9], [0, 2, 1, 6], 6, 6, None),
    "starts that go beyond the tokens": ([100, 40, 9], [0, 1, 2, 9], 6, 8, None),
    "more new tokens than promised": ([100, 40, 9], [0, 1, 2, 6], 6, 3, [0, 1]),
    "a length beyond the table": ([100, 5000, 9], [0, 1, 2, 6], 6, 4, [0, 2, 3, 4, 5]),
    "a length below zero": ([100, -3, 9], [0, 1, 2, 6], 6, 4, [0, 2, 3, 4, 5]),
    "a length beyond the table, nothing new of it": ([100, 5000, 9], [0, 1, 1, 6], 6, 5, [0, 1, 2, 3, 4, 5]),
}


def fresh(group):
    return Case([100, 40, 9], [2, 2, 2], 2, group).fill()


def batch_of(c, lengths, starts, tokens, max_new, max_length):
    i32 = dict(dtype=torch.int32, device="cuda")
    return binding.PagedBatch(c.table, torch.tensor(lengths, **i32), torch.tensor(starts, **i32), tokens, max_new, max_length)


# 2 query rows a token and kv head stream, in parts by the grid or (from what the longest length says) by the lengths; 40 take tiles
@pytest.mark.parametrize("group,max_length", [(2, 128), (2, 1 << 20), (40, 128)])
@pytest.mark.parametrize("wrong", WRONG)
def test_an_attend_says_so_itself(wrong, group, max_length):
    lengths, starts, tokens, max_new, owned = WRONG[wrong]
    c = fresh(group)
    rng = np.random.default_rng(2)
    Qh = po.to_bf16(rng.standard_normal((tokens, 2 * group, 128)).astype(np.float32))
    O, lse = torch.full((tokens, 2 * group, 128), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((tokens, 2 * group), 7.0, device="cuda")
    c.kv.scalekv_paged_attend(c.layer, batch_of(c, lengths, starts, tokens, max_new, max_length), torch.from_numpy(Qh).cuda().bfloat16(), O, lse)
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()
    if owned is None:
        return
    got, got_lse = O.float().cpu().numpy(), lse.cpu().numpy()
    for b in range(3):
        n, length = starts[b + 1] - starts[b], lengths[b]
        if starts[b] < 0 or n < 1 or n > max_new or not 0 <= length <= c.lengths[b]:
            continue
        k, v = c.rows(c.K, b)[:length], c.rows(c.V, b)[:length]
        seen = po.visible(n, length, True, 0, 0)
        for h in range(2 * group):
            want, _, A, _ = po.attend(Qh[starts[b]:starts[b + 1], h], k[:, h // group], v[:, h // group], seen, 128 ** -0.5)
            assert (np.abs(got[starts[b]:starts[b + 1], h] - want) <= 2.0 ** -8 * (np.abs(want) + A) + 2.0 ** -12 * A).all(), (b, h)
    if not wrong.startswith(("a length", "more", "a first start below")):
        rest = [t for t in range(tokens) if t not in owned]
        assert (got[rest] == 7).all() and (got_lse[rest] == 7).all()


@pytest.mark.parametrize("wrong", [w for w in WRONG if not w.startswith(("more new", "a length beyond the table, nothing"))])
@pytest.mark.parametrize("call", ["write", "read"])
def test_a_write_or_read_says_so_itself(wrong, call):
    lengths, starts, tokens, max_new, _ = WRONG[wrong]
    c = fresh(1)
    batch = batch_of(c, lengths, starts, tokens, max_new, 128)
    if call == "read":
        c.kv.scalekv_paged_read(c.layer, batch)
    else:
        x = torch.ones(tokens, 2, 128, device="cuda")
        c.kv.scalekv_paged_write(c.layer, batch, x, x)
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()


@pytest.mark.parametrize("group,max_length", [(2, 128), (2, 1 << 20), (40, 128)])
def test_a_batch_in_order_is_not_reported(group, max_length):
    c = fresh(group)
    for starts, tokens in (([0, 2, 4, 6], 6), ([0, 0, 6, 6], 6), ([0, 0, 0, 1], 1), ([0, 6, 6, 6], 6)):
        batch = batch_of(c, c.lengths, starts, tokens, 6, max_length)
        c.kv.scalekv_paged_attend(c.layer, batch, torch.zeros(tokens, 2 * group, 128, device="cuda", dtype=torch.bfloat16))
        c.kv.scalekv_paged_read(c.layer, batch)
    c.kv.scalekv_paged_sync()
