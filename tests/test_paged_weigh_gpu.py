"""Attention summed up entry by entry, and eviction by it, against plain implementations.

Tolerances of a sum: every p = exp(y - lse) is off by what its exponent is, 2 (d + 4) 2^-24 of Y = scale sum |q k| for the product and 2^-21 of 1 + |lse| + |y| for scaling, the
difference in base 2 and the exponential; n + 2 sums round by 2^-24 of their result each.  Eviction moves bits: nothing is off."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case
from tests.test_paged_tree_gpu import pool_rows

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(c, causal=True, window=0, n_sink=0, decay=1.0, scale=0.0, lse=None, max_length=None, Q=None):
    T, k1 = sum(c.new), scale or 1 / math.sqrt(c.d)
    Qd = torch.from_numpy(c.Q).cuda().bfloat16() if Q is None else Q
    if lse is None:
        lse = torch.empty(T, c.H * c.G, device="cuda")
        c.kv.scalekv_paged_attend(c.layer, c.batch(max_length=max_length), Qd, None, lse, causal, window, n_sink, scale)
    old = torch.rand(c.kv.n_pages, c.H, c.page, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * 3
    weights = old.clone()
    c.kv.scalekv_paged_weigh(c.layer, c.batch(max_length=max_length), Qd, lse, weights, causal, window, n_sink, decay, scale)
    c.kv.scalekv_paged_sync()
    again = old.clone()
    c.kv.scalekv_paged_weigh(c.layer, c.batch(max_length=max_length), Qd, lse, again, causal, window, n_sink, decay, scale)
    assert torch.equal(again, weights)                                    # sums have one order
    got, want, lse, table = weights.cpu().numpy(), old.cpu().numpy().astype(np.float64), lse.cpu().numpy(), c.table.cpu().numpy()
    tol = np.zeros(got.shape)
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        seen = po.visible(n, length, causal, window, n_sink)
        some, t0 = seen.any(0), sum(c.new[:b])
        pos = np.arange(length)
        page, row = table[b, pos // c.page], pos % c.page
        fade = np.where(some, np.where(pos < length - n, np.float64(np.float32(decay)), 0.0), 1.0) if n else np.ones(length)
        for h in range(c.H):
            k = c.rows(c.K, b)[:, h]
            w = want[page, h, row] * fade
            off = np.where(some, 2.0 ** -23 * np.abs(w), 0)
            for g in range(h * c.G, (h + 1) * c.G):
                s, SY, SE = po.attention_got(c.Q[t0:t0 + n, g], k, lse[t0:t0 + n, g], seen, k1)
                w = w + s
                off = off + 2 * (c.d + 4) * 2.0 ** -24 * SY + 2.0 ** -21 * SE + (n * c.G + 2) * 2.0 ** -24 * s
            want[page, h, row], tol[page, h, row] = w, off
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
    return weights


CASES = [  # lengths, new, kv heads, group, page
    ([1], [1], 1, 1, 16),
    ([40, 17, 0, 300], [1, 1, 0, 1], 2, 4, 16),
    ([200, 131, 64], [8, 0, 3], 2, 1, 32),
    ([300, 33], [4, 3], 3, 4, 64),
    ([450, 31], [31, 31], 1, 1, 16),
    ([140, 97, 5], [33, 12, 5], 2, 1, 64),
    ([500, 129, 640], [64, 100, 1], 1, 4, 64),
    ([700, 257], [70, 257], 2, 5, 128),
    ([1500], [600], 1, 3, 16),
]


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,new,heads,group,page", CASES)
def test_weights(store, d, lengths, new, heads, group, page):
    c = Case(lengths, new, heads, group, d, store, page).fill()
    check(c)
    check(c, decay=0.75, scale=0.2)


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("lengths,new,heads,group", [([400, 90], [1, 1], 2, 2), ([400, 90], [7, 5], 1, 1), ([700, 390], [150, 64], 2, 3)])
@pytest.mark.parametrize("causal,window,n_sink", [(True, 50, 3), (False, 0, 0), (False, 70, 20), (True, 1, 0), (True, 10000, 4)])
def test_masks(store, lengths, new, heads, group, causal, window, n_sink):
    c = Case(lengths, new, heads, group, 64, store).fill()
    check(c, causal, window, n_sink, decay=0.5)
    check(c, causal, window, n_sink)


@pytest.mark.parametrize("new", [[3], [90]])
def test_rows_that_saw_nothing_pay_nothing(new):
    c = Case([200], new, 2, 2, 64).fill()
    lse = torch.zeros(new[0], 4, device="cuda") + 5
    lse[1::2] = -float("inf")
    check(c, lse=lse)
    weights = check(c, lse=torch.full_like(lse, -float("inf")))
    assert torch.isfinite(weights).all()


@pytest.mark.parametrize("new", [[5], [80]])
def test_queries_ahead_of_the_cache(new):
    c = Case([new[0] - 3], new, 1, 1, 64).fill()          # more tokens than entries: the first ones see nothing
    check(c)
    c = Case([0, 30], [new[0], 2], 1, 1, 64).fill()
    check(c)


@pytest.mark.parametrize("max_length", [1, 100, 100000])
def test_max_length_only_sizes_launches(max_length):
    check(Case([3000, 10], [1, 1], 1, 2, 64).fill(), max_length=max_length)
    check(Case([900, 60], [50, 40], 1, 2, 64).fill(), max_length=max_length)


@pytest.mark.parametrize("new", [[1], [60]])
def test_hidden_entries_may_hold_anything(new):
    """What a window hides has pages that are somebody else's: their weights are left alone."""
    c = Case([400], new, 1, 1, 64, page=16).fill()
    lo = (400 - new[0] - 50 + 1) // 16
    weights = check(c, window=50, decay=0.5)
    c.table[0, 1:lo] = -3
    old = torch.zeros_like(weights)
    lse = torch.full((new[0], 1), 4.0, device="cuda")
    c.kv.scalekv_paged_weigh(c.layer, c.batch(), torch.from_numpy(c.Q).cuda().bfloat16(), lse, old, window=50, decay=0.5)
    c.kv.scalekv_paged_sync()


def test_pages_out_of_range_are_told():
    for new in (1, 60):
        c = Case([100], [new], 1, 1, 64).fill()
        c.table[0, 2] = c.kv.n_pages
        weights = torch.zeros(c.kv.n_pages, 1, 16, device="cuda")
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), torch.from_numpy(c.Q).cuda().bfloat16(), torch.full((new, 1), 3.0, device="cuda"), weights)
        with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
            c.kv.scalekv_paged_sync()
        assert int((weights > 0).sum()) == 84


def test_refused_weighings():
    c = Case([100], [4], 2, 2, 64).fill()
    Q, lse, w = torch.from_numpy(c.Q).cuda().bfloat16(), torch.zeros(4, 4, device="cuda"), torch.zeros(c.kv.n_pages, 2, 16, device="cuda")
    for args in ((Q, lse[:3], w), (Q, lse.double(), w), (Q, lse, w[1:]), (Q, lse, w.transpose(1, 2)), (Q, lse, w.half()), (Q.float(), lse, w), (Q, lse.t(), w), (Q, lse, w.cpu())):
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_weigh(c.layer, c.batch(), *args)
    for decay in (-0.1, 1.5, float("nan")):
        with pytest.raises(binding.ScaleKVError, match="decay"):
            c.kv.scalekv_paged_weigh(c.layer, c.batch(), Q, lse, w, decay=decay)
    with pytest.raises(binding.ScaleKVError, match="heads"):
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), Q[:, :3], lse[:, :3].contiguous(), w)
    with pytest.raises(ValueError, match="window"):
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), Q, lse, w, window=-1)
    with pytest.raises(binding.ScaleKVError, match="aligned"):
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), Q, lse, torch.zeros(w.numel() + 1, device="cuda")[1:].view(w.shape))
    c.kv.scalekv_paged_sync()
    assert not w.any()


# ---- eviction ----------------------------------------------------------------------------------------------------------------------
def evict(lengths, keep, heads=2, d=64, store="q8", page=16, n_sink=0, n_recent=0, kind="random", seed=0, max_length=None, give=True):
    c = Case(lengths, [0] * len(lengths), heads, 1, d, store, page, seed=seed, spare=sum(-(-max(k, 0) // page) for k in keep) + 2)
    g = torch.Generator(device="cuda").manual_seed(seed + 7)
    c.kv.pool.copy_(torch.randint(0, 256, c.kv.pool.shape, generator=g, device="cuda", dtype=torch.uint8))
    used = set(c.table.cpu().numpy().ravel().tolist())
    free = [p for p in range(c.kv.n_pages) if p not in used]
    to = np.full((len(lengths), max(1, max(-(-max(k, 0) // page) for k in keep))), -1, np.int32)
    for b, k in enumerate(keep):
        for i in range(-(-max(k, 0) // page)):
            to[b, i] = free.pop()
    u = torch.rand(c.kv.n_pages, heads, page, generator=g, device="cuda")
    weights = {"random": u, "equal": torch.full_like(u, 0.25), "few": (u * 5).floor(), "signs": torch.where(u < 0.5, -u, u) * 1e30, "tiny": u * 1e-42,
               "odd": torch.where(u < 0.2, float("nan"), torch.where(u < 0.4, -float("inf"), torch.where(u < 0.5, float("inf"), torch.where(u < 0.7, -0.0, 0.0))))}[kind].contiguous()
    old, before = weights.clone(), [x.clone() for x in pool_rows(c)]
    most = max(max(keep), 1)
    kept = torch.full((len(lengths), heads, most + 3), -9, dtype=torch.int32, device="cuda") if give else None
    dev = dict(dtype=torch.int32, device="cuda")
    kept = c.kv.scalekv_paged_evict(c.layer, c.batch(max_length=max_length), torch.from_numpy(to).cuda(), torch.tensor(keep, **dev), weights, n_sink, n_recent, kept)
    c.kv.scalekv_paged_sync()
    got, table, want_w = kept.cpu().numpy(), c.table.cpu().numpy(), old.clone()
    want = [x.clone() for x in before]
    for b, length in enumerate(lengths):
        pos = np.arange(length)
        for h in range(heads):
            w = old.cpu().numpy()[table[b, pos // page], h, pos % page]
            stay = po.stays(w, keep[b], n_sink, n_recent)
            assert got[b, h, :len(stay)].tolist() == stay.tolist(), (b, h)
            assert (got[b, h, len(stay):] == (-9 if give else -1)).all()
            src = torch.from_numpy(stay).cuda()
            dst = torch.arange(len(stay), device="cuda")
            sp, tp = c.table[b].long()[src // page], torch.from_numpy(to[b]).cuda().long()[dst // page]
            for x, y in zip(want, before):
                x[c.layer, tp, h, dst % page] = y[c.layer, sp, h, src % page]
            want_w[tp, h, dst % page] = old[sp, h, src % page]
    for x, y in zip(want, pool_rows(c)):
        assert torch.equal(x, y)
    assert torch.equal(want_w.view(torch.int32), weights.view(torch.int32))


@pytest.mark.parametrize("kind", ["random", "equal", "few", "signs", "tiny", "odd"])
@pytest.mark.parametrize("lengths,keep,n_sink,n_recent", [([1], [1], 0, 0), ([70, 0, 333, 16], [20, 5, 40, 16], 4, 10), ([200, 100], [0, 99], 0, 0), ([513], [64], 0, 64),
                                                          ([90], [10], 300, 300), ([90], [12], 5, 300), ([1000, 2000], [7, 1500], 1, 0)])
def test_evictions(kind, lengths, keep, n_sink, n_recent):
    evict(lengths, keep, n_sink=n_sink, n_recent=n_recent, kind=kind)


@pytest.mark.parametrize("d,store,page,heads", [(128, "q8", 64, 1), (128, "bf16", 32, 3), (64, "bf16", 128, 5)])
def test_evictions_of_other_caches(d, store, page, heads):
    evict([400, 777, 3], [123, 640, 2], heads, d, store, page, 2, 30, give=False)


@pytest.mark.parametrize("length,heads,kind", [(5000, 1, "random"), (40000, 2, "few"), (70001, 1, "random"), (400000, 1, "few"), (400000, 1, "equal"), (60000, 33, "random")])
def test_long_evictions(length, heads, kind):
    """Clusters of CTAs, and stretches that find no room in shared memory."""
    evict([length, length // 3], [length // 10, length // 4], heads, 64, "q8", 128, 4, 100, kind)


@pytest.mark.parametrize("max_length", [1, 1000000])
def test_max_length_only_sizes_an_eviction(max_length):
    evict([9000], [800], 1, max_length=max_length)


def test_wrong_evictions_are_told():
    dev = dict(dtype=torch.int32, device="cuda")
    for keep, to, most, changed in (([-1, 5], None, 16, 1), ([17, 5], None, 16, 1), ([20, 5], None, 40, 1), ([16, 5], 99, 16, 1), ([16, 5], -1, 16, 1), ([16, 5], None, 16, 2)):
        c = Case([60, 30], [0, 0], 1, 1, 64, spare=4)
        free = [p for p in range(c.kv.n_pages) if p not in c.table.cpu().numpy().ravel().tolist()]
        table = torch.tensor([[free[0] if to is None else to], [free[1]]], **dev)
        weights = torch.rand(c.kv.n_pages, 1, 16, device="cuda")
        old = weights.clone()
        kept = torch.full((2, 1, most), -1, **dev)
        c.kv.scalekv_paged_evict(c.layer, c.batch(), table, torch.tensor(keep, **dev), weights, kept=kept)
        if changed == 2:
            c.kv.scalekv_paged_sync()
        else:
            with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
                c.kv.scalekv_paged_sync()
        assert [bool((weights != old)[p].any()) for p in free[:2]] == [changed == 2, True]
        assert not (weights != old)[[p for p in range(c.kv.n_pages) if p not in free[:2]]].any()


def test_refused_evictions():
    c = Case([60], [0], 2, 1, 64, spare=4)
    dev = dict(dtype=torch.int32, device="cuda")
    to, keep, w, kept = torch.zeros(1, 2, **dev), torch.zeros(1, **dev), torch.zeros(c.kv.n_pages, 2, 16, device="cuda"), torch.zeros(1, 2, 20, **dev)
    for args in ((to[0], keep, w), (to, keep.long(), w), (to, keep, w[:, :1]), (to, torch.zeros(2, **dev), w), (to.cpu(), keep, w)):
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_evict(c.layer, c.batch(), *args)
    for k in (kept[:, :1], kept.float(), kept[0], kept.transpose(1, 2)):
        with pytest.raises(ValueError, match="kept"):
            c.kv.scalekv_paged_evict(c.layer, c.batch(), to, keep, w, kept=k)
    for sink, recent in ((-1, 0), (0, -1), (2 ** 31, 0)):
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_evict(c.layer, c.batch(), to, keep, w, sink, recent, kept)
    with pytest.raises(binding.ScaleKVError, match="layer"):
        c.kv.scalekv_paged_evict(5, c.batch(), to, keep, w)
    with pytest.raises(binding.ScaleKVError, match="aligned"):
        c.kv.scalekv_paged_evict(c.layer, c.batch(), to, keep, torch.zeros(w.numel() + 1, device="cuda")[1:].view(w.shape))
    c.kv.scalekv_paged_sync()
