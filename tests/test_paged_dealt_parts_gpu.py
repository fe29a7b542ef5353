"""Streaming launches whose parts are dealt out on the device by the lengths, in both ways (equal parts of every sequence, equal shares of all
steps), with 1-8, 9-16 and 17-32 query rows, against fp64.  Which way a launch goes is asked of the rules themselves.  Tolerances as derived in
test_paged_gpu.py."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po
from tests import stream_rule as sr
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def spread(n, longest, seed):
    return [int(x) for x in np.random.default_rng(seed).integers(longest * 2 // 5, longest, n)]


# one long sequence among short ones: shares; sequences of about the same length: parts; some empty, some without new tokens
UNEVEN = [9000] + spread(12, 400, 1) + [0, 1, 17, 5] + spread(9, 900, 2) + [2500]
EVEN = spread(30, 1500, 3) + [0, 3]


def way(c, d, store, rows, keys):
    """What the rules make of this call: "grid", "parts" or "shares"."""
    n_sm = torch.cuda.get_device_properties(0).multi_processor_count
    slots, tiles = sr.slots(d, store, rows, n_sm), 1 if rows <= 16 else 2
    n_seqs, heads = len(c.lengths), c.H * tiles
    _, most = sr.cut(slots, n_seqs, n_seqs * heads, sum(c.new) * c.H * c.G, keys, n_sm)
    if not most:
        return "grid"
    steps = [max(-(-length // 16), 1) if n else 0 for n, length in zip(c.new, c.lengths)]
    return "shares" if sr.deal(sum(steps) * heads, max(steps), n_seqs * heads, slots, most)[1] else "parts"


def check(c, keys, window=0, n_sink=0):
    Q = torch.from_numpy(c.Q).cuda().bfloat16()
    lse = torch.full((sum(c.new), c.H * c.G), 7.0, device="cuda")
    batch = c.batch(max_length=keys)
    O = c.kv.scalekv_paged_attend(c.layer, batch, Q, lse=lse, window=window, n_sink=n_sink)
    again = c.kv.scalekv_paged_attend(c.layer, batch, Q, window=window, n_sink=n_sink)      # (the counters are back at zero)
    c.kv.scalekv_paged_sync()
    assert torch.equal(O, again)
    O, t0 = O.double(), 0
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        got, got_lse, q = O[t0:t0 + n], lse[t0:t0 + n], Q[t0:t0 + n].double()
        t0 += n
        if not n:
            continue
        k, v = (torch.from_numpy(c.rows(x, b)).cuda().double().repeat_interleave(c.G, 1) for x in (c.K, c.V))
        seen = torch.from_numpy(po.visible(n, length, True, window, n_sink)).cuda()[None]
        y = (torch.einsum("nhd,lhd->hnl", q, k) / math.sqrt(c.d)).masked_fill(~seen, -math.inf)
        empty = ~seen[0].any(1)
        p = torch.nan_to_num(torch.softmax(y, -1))
        want, A = torch.einsum("hnl,lhd->nhd", p, v), torch.einsum("hnl,lhd->nhd", p, v.abs())
        assert bool(((got - want).abs() <= 2.0 ** -8 * (want.abs() + A) + 2.0 ** -12 * A).all()), b
        assert bool((got_lse[empty] == -math.inf).all())
        if length == 0 or bool(empty.all()):
            continue
        Y = (torch.einsum("nhd,lhd->hnl", q.abs(), k.abs()) / math.sqrt(c.d)).masked_fill(~seen, 0).amax(-1).T
        want_lse = torch.logsumexp(y, -1).T
        tol = 2 * (c.d + 4) * 2.0 ** -24 * Y + 2.0 ** -18 * (1 + want_lse.abs())
        assert bool(((got_lse - want_lse).abs() <= tol)[~empty].all()), b


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 128), ("q8", 64), ("bf16", 64)])
@pytest.mark.parametrize("new,group", [(1, 4), (3, 4), (2, 8), (6, 4), (4, 8)])
@pytest.mark.parametrize("lengths,want", [(UNEVEN, "shares"), (EVEN, "parts")])
def test_both_ways(lengths, want, new, group, store, d):
    """The longest length is promised longer than it is, which sizes the launch and nothing else."""
    counts = [0 if b % 7 == 5 else 1 + b % new for b in range(len(lengths))]
    counts[0] = new
    c = Case(lengths, counts, 2, group, d, store, page=64)
    assert way(c, d, store, new * group, 1 << 20) == want
    check(c.fill(), 1 << 20)


@pytest.mark.parametrize("new,group", [(1, 4), (4, 8)])
def test_with_a_window(new, group):
    for lengths in (UNEVEN, EVEN):
        c = Case(lengths, [new] * len(lengths), 2, group, 128, "q8", page=16).fill()
        check(c, 1 << 20, window=300, n_sink=5)                     # (short: the keys that count are few, and the grid cuts them)
        check(c, 1 << 20, window=20000, n_sink=5)


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 128), ("q8", 64)])
def test_as_long_as_they_are(store, d):
    """Lengths that take this way by themselves."""
    lengths = spread(40, 9600, 4) + [9600, 0, 33]
    c = Case(lengths, [0 if b == 9 else 1 for b in range(len(lengths))], 2, 4, d, store, page=128)
    assert way(c, d, store, 4, max(lengths)) in ("parts", "shares")
    check(c.fill(), max(lengths))


def test_more_items_than_places():
    """Several parts to a CTA: more sequences and heads than CTAs in the launch."""
    lengths = spread(300, 400, 5) + [2000]
    c = Case(lengths, [1] * len(lengths), 4, 2, 128, "q8", page=64)
    assert len(lengths) * 4 > sr.slots(128, "q8", 2) and way(c, 128, "q8", 2, 1 << 20) in ("parts", "shares")
    check(c.fill(), 1 << 20)
