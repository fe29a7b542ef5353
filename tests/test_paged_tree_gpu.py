"""Attention of drafted tokens, and drafts accepted, against plain implementations.  Tolerances as in test_paged_gpu.py; accepted rows are the same bits."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def tree(rng, n):
    """What the tokens of a random tree see: their ancestors and themselves."""
    sees = []
    for i in range(n):
        parent = int(rng.integers(max(-1, i - 8), i)) if i else -1
        sees.append((sees[parent] if parent >= 0 else []) + [i])
    return sees


def draft(c, sees, words=None, scale=0.0, Q=None, O=None, more=0):
    words = words or -(-max(c.new + [1]) // 32)
    bits = torch.from_numpy(np.concatenate([po.draft_bits(s, words + more) for s in sees])).cuda()
    T = sum(c.new)
    Qd = torch.from_numpy(c.Q).cuda().bfloat16() if Q is None else Q
    lse = torch.full((T, c.H * c.G), 7.0, device="cuda")
    O = c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Qd, bits, O, lse, scale)
    c.kv.scalekv_paged_sync()
    return O, lse


def check(c, sees, scale=0.0, **more):
    O, lse = draft(c, sees, scale=scale, **more)
    got, got_lse, k1 = O.float().cpu().numpy(), lse.cpu().numpy(), scale or 1 / math.sqrt(c.d)
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        seen = po.draft_visible(sees[b], length)
        t0 = sum(c.new[:b])
        k, v = c.rows(c.K, b), c.rows(c.V, b)
        for h in range(c.H * c.G):
            want, want_lse, A, Y = po.attend(c.Q[t0:t0 + n, h], k[:, h // c.G], v[:, h // c.G], seen, k1)
            x, g = got[t0:t0 + n, h], got_lse[t0:t0 + n, h]
            empty = ~seen.any(1)
            assert (g[empty] == -np.inf).all() and (x[empty] == 0).all()
            assert (np.abs(x - want) <= 2.0 ** -8 * (np.abs(want) + A) + 2.0 ** -12 * A + 1e-30).all(), (b, h)
            tol = 2 * (c.d + 4) * 2.0 ** -24 * Y + 2.0 ** -18 * (1 + np.abs(want_lse))
            assert (np.abs(g[~empty] - want_lse[~empty]) <= tol[~empty]).all(), (b, h)


CASES = [  # lengths, new, kv heads, group, page
    ([1], [1], 1, 1, 16),
    ([17, 40, 0, 5], [8, 0, 0, 5], 2, 1, 16),
    ([200, 131, 64], [8, 7, 3], 2, 2, 32),
    ([300, 31], [31, 31], 1, 1, 16),
    ([140, 97], [33, 12], 2, 1, 64),
    ([500, 129], [64, 64], 1, 4, 64),
    ([700], [70], 2, 5, 128),
    ([150, 260], [129, 33], 1, 3, 16),
    ([3000], [40], 1, 8, 64),
]


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,new,heads,group,page", CASES)
def test_trees(store, d, lengths, new, heads, group, page):
    c = Case(lengths, new, heads, group, d, store, page).fill()
    check(c, [tree(c.rng, n) for n in new])


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 64)])
@pytest.mark.parametrize("lengths,new,heads,group", [
    ([6000, 300, 2000], [70, 40, 64], 2, 2),                  # one item of a pair of tiles beside singles
    ([4000], [65], 1, 8),                                     # one sequence, three items, one of them short
    ([5000, 0, 33, 700, 40, 1300], [40, 0, 33, 9, 0, 64], 1, 1),      # sequences without a draft between others
    ([40] * 40 + [3000], [33] * 41, 2, 1),                    # many short ones and a long one
    ([200] * 170, [36] * 170, 1, 1),                          # more items than CTAs
])
def test_ragged_drafts(store, d, lengths, new, heads, group):
    c = Case(lengths, new, heads, group, d, store, 64).fill()
    sees = [tree(c.rng, n) for n in new]
    check(c, sees)
    again = draft(c, sees)
    assert all(torch.equal(x, y) for x, y in zip(draft(c, sees), again))


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("new,group", [([6, 3], 1), ([31, 6], 1), ([50, 9], 3)])
def test_any_bits(store, new, group):
    """Bits that are no tree: tokens that see later ones, or nothing of the draft, a draft with nothing before it, one longer than the cache."""
    c = Case([new[0] + 57, new[1]], new, 2, group, 64, store).fill()
    sees = [[[j for j in range(n) if c.rng.random() < 0.3] for _ in range(n)] for n in new]
    sees[0][0], sees[1][0], sees[1][-1] = [], [], list(range(new[1]))
    check(c, sees)
    check(c, sees, more=2, scale=0.3)
    c = Case([new[0] - 2], [new[0]], 2, group, 64, store).fill()          # (its first two tokens are nowhere in the cache)
    check(c, [sees[0]])


def test_a_chain_is_a_causal_mask():
    for new, group in (([5, 2], 1), ([40, 64], 2)):
        c = Case([333, 90], new, 2, group, 128).fill()
        O, lse = draft(c, [[list(range(i + 1)) for i in range(n)] for n in new])
        want_lse = torch.empty_like(lse)
        want = c.kv.scalekv_paged_attend(c.layer, c.batch(), torch.from_numpy(c.Q).cuda().bfloat16(), None, want_lse)
        c.kv.scalekv_paged_sync()
        assert torch.equal(O, want) and torch.equal(lse, want_lse)


def test_bits_behind_the_draft_count_for_nothing():
    c = Case([100, 60], [9, 4], 2, 1, 64).fill()
    sees = [tree(c.rng, n) for n in c.new]
    bits = np.concatenate([po.draft_bits(s, 1) for s in sees]).view(np.uint32)
    bits[:9] |= np.uint32(0xffffffff) << np.uint32(9)
    bits[9:] |= np.uint32(0xffffffff) << np.uint32(4)
    want, want_lse = draft(c, sees)
    lse = torch.empty_like(want_lse)
    Q = torch.from_numpy(c.Q).cuda().bfloat16()
    O = c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Q, torch.from_numpy(bits.view(np.int32)).cuda(), None, lse)
    c.kv.scalekv_paged_sync()
    assert torch.equal(O, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("new,group", [([7], 1), ([70], 1)])
def test_hidden_keys_may_hold_anything(new, group):
    """K of a drafted token that others do not see, and with codes its V: NaN reaches those alone that see it."""
    c = Case([new[0] + 130], new, 1, group, 64, "q8").fill()
    K = c.K.copy()
    K[-1, 0, 3] = np.nan
    n = new[0]
    c.kv.scalekv_paged_write(c.layer, c.batch([n]), torch.from_numpy(K[-n:]).cuda(), torch.from_numpy(K[-n:]).cuda())
    sees = [[[i] for i in range(n)]]
    O, lse = draft(c, sees)
    assert torch.isfinite(O[:-1].float()).all() and torch.isfinite(lse[:-1]).all() and torch.isnan(lse[-1]).all() and torch.isnan(O[-1].float()).all()


def test_refused_drafts():
    c = Case([100], [40], 2, 1, 64).fill()
    Q, bits = torch.from_numpy(c.Q).cuda().bfloat16(), torch.zeros(40, 2, dtype=torch.int32, device="cuda")
    for wrong in (bits[:39], bits.long(), bits.cpu(), bits[:, 0], bits.t().contiguous().t()):
        with pytest.raises(ValueError, match="tree"):
            c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Q, wrong)
    with pytest.raises(binding.ScaleKVError, match="bit"):
        c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Q, bits[:, :1].contiguous())
    with pytest.raises(TypeError):
        c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Q, None)
    with pytest.raises(binding.ScaleKVError, match="softmax_scale"):
        c.kv.scalekv_paged_attend_tree(c.layer, c.batch(), Q, bits, softmax_scale=-1.0)
    with pytest.raises(binding.ScaleKVError, match="layer"):
        c.kv.scalekv_paged_attend_tree(-1, c.batch(), Q, bits)
    c.kv.scalekv_paged_sync()


# ---- accepted tokens ---------------------------------------------------------------------------------------------------------------
def pool_rows(c):
    """Views of the pool's four parts (two for bf16 rows), [layer, page, head, row, bytes]."""
    rows = c.kv.pool.numel() // (2 * (c.d + 4) if c.store == "q8" else 4 * c.d)
    parts = [rows * c.d] * 2 + [rows * 4] * 2 if c.store == "q8" else [rows * 2 * c.d] * 2
    return [x.view(c.kv.n_layers, c.kv.n_pages, c.H, c.page, -1) for x in torch.split(c.kv.pool, parts)]


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layer", [None, 1])
@pytest.mark.parametrize("lengths,new,heads,page", [([8], [8], 1, 16), ([40, 3, 200, 90], [33, 0, 150, 1], 3, 16), ([300, 77], [200, 77], 9, 64)])
def test_accepted_rows_move(store, d, layer, lengths, new, heads, page):
    c = Case(lengths, new, heads, 1, d, store, page, layers=3, layer=1)
    g = torch.Generator(device="cuda").manual_seed(3)
    c.kv.pool.copy_(torch.randint(0, 256, c.kv.pool.shape, generator=g, device="cuda", dtype=torch.uint8))
    counts = [int(c.rng.integers(0, n + 1)) for n in new]
    counts[0] = new[0] // 2 + 1
    paths = [sorted(c.rng.choice(n, k, replace=False).tolist()) for n, k in zip(new, counts)]
    most = max(counts) + 2
    path = torch.tensor([p + [-5] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    want = [x.clone() for x in pool_rows(c)]
    table = c.table.cpu()
    for b, p in enumerate(paths):
        first = lengths[b] - new[b]
        for x, y in zip(want, pool_rows(c)):
            for l in range(3) if layer is None else [layer]:
                for i, j in enumerate(p):
                    x[l, table[b, (first + i) // page], :, (first + i) % page] = y[l, table[b, (first + j) // page], :, (first + j) % page]
    c.kv.scalekv_paged_accept(c.batch(), path, torch.tensor(counts, dtype=torch.int32, device="cuda"), layer)
    c.kv.scalekv_paged_sync()
    for x, y in zip(want, pool_rows(c)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("path,count,moved", [([3, 2, 5], 3, 1), ([1, 8, 9], 3, 1), ([-1, 2, 3], 3, 0), ([2, 2, 3], 3, 1), ([1, 2, 3], 4, 0), ([1, 2, 3], -1, 0), ([1, 4, 7], 3, 3)])
def test_wrong_paths_are_told(path, count, moved):
    c = Case([20], [8], 2, 1, 64)
    c.kv.pool.copy_(torch.arange(c.kv.pool.numel(), device="cuda").remainder(251).to(torch.uint8))
    want = [x.clone() for x in pool_rows(c)]
    t = c.table.cpu()
    for x, y in zip(want, pool_rows(c)):
        for i in range(moved):
            x[:, t[0, (12 + i) // 16], :, (12 + i) % 16] = y[:, t[0, (12 + path[i]) // 16], :, (12 + path[i]) % 16]
    dev = dict(dtype=torch.int32, device="cuda")
    c.kv.scalekv_paged_accept(c.batch(), torch.tensor([path], **dev), torch.tensor([count], **dev))
    if moved == 3:
        c.kv.scalekv_paged_sync()
    else:
        with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
            c.kv.scalekv_paged_sync()
    for x, y in zip(want, pool_rows(c)):
        assert torch.equal(x, y)


def test_refused_paths():
    c = Case([20, 9], [8, 4], 2, 1, 64)
    dev = dict(dtype=torch.int32, device="cuda")
    path, counts = torch.zeros(2, 3, **dev), torch.zeros(2, **dev)
    for p, k in ((path[:1], counts), (path.long(), counts), (path, counts[:1]), (path, counts.float()), (path.cpu(), counts), (path[0], counts)):
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_accept(c.batch(), p, k)
    for layer in (2, -1, -2, 2 ** 32):
        with pytest.raises(binding.ScaleKVError, match="layer"):
            c.kv.scalekv_paged_accept(c.batch(), path, counts, layer)
    c.kv.scalekv_paged_accept(c.batch(), path[:, :0], counts)             # nothing to accept
    c.kv.scalekv_paged_sync()
