"""Drafts, tokens and evictions one behind the other through pipeline alone: the accepted tokens' sums are those of tokens that came in a step of their own."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding, pipeline

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
LAYERS, H, G, D, PAGE, PAGES = 2, 2, 2, 64, 16, 120
ROTARY = binding.Rotary([8, 12, 12])


class Server:
    def __init__(self, store, n_seqs=3):
        self.kv = binding.PagedKV(LAYERS, PAGES, H, D, store=store, page_tokens=PAGE)
        self.kv.pool.fill_(255)
        self.seqs = pipeline.Sequences(PAGES, PAGE, n_seqs, 600)
        self.weights = torch.full((LAYERS, PAGES, H, PAGE), float("nan"), device="cuda")

    def sums(self, l, b):
        pos = np.arange(self.seqs.lengths[b])
        return self.weights[l].cpu().numpy()[np.array(self.seqs.table[b])[pos // PAGE].astype(int), :, pos % PAGE]


def rows_of(rng, T, rotary, shared):
    """Rows of every layer; without `rotary` as attends take them.  shared: every layer's are put into the same tensors."""
    given = [[torch.from_numpy(rng.standard_normal((T, n, D)).astype(np.float32)).cuda().to(torch.float32 if rotary else torch.bfloat16) for n in (H * G, H, H)] for _ in range(LAYERS)]
    buffer = [torch.empty_like(x) for x in given[0]]

    def rows(l):
        return [b.copy_(x) for b, x in zip(buffer, given[l])] if shared else given[l]

    return rows


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("rotary,shared", [(ROTARY, False), (None, False), (None, True)])
def test_drafts_leave_sums_that_an_eviction_can_rank(store, rotary, shared):
    rng = np.random.default_rng(4)
    s, by_hand = Server(store), Server(store)

    def positions(T):
        return torch.from_numpy(rng.integers(0, 5000, (3, T)).astype(np.int32)).cuda() if rotary else None

    for turn in range(2):
        for new in ([70, 7, 33], [1, 1, 0]):
            rows, at = rows_of(rng, sum(new), rotary, shared), positions(sum(new))
            for x in (s, by_hand):
                x.seqs.extend(new)
                pipeline.token_step(x.kv, x.seqs.batch(new), rows, rotary=rotary, positions=at, weights=x.weights, decay=0.9)
        parents = [[-1, 0, 0, 2, 3, 3, -1], [-1], [-1, 0, 1][:3 * turn]]
        paths = [[0, 2, 3, 5], [], [0, 1][:2 * turn]]
        rows, at, n = rows_of(rng, sum(map(len, parents)), rotary, shared), positions(sum(map(len, parents))), [len(p) for p in paths]
        out, got = pipeline.draft_step(s.kv, s.seqs, parents, rows, lambda out: paths, rotary, at, weights=s.weights, decay=0.9)
        assert got == paths and len(out) == LAYERS
        # by hand: the rows of the accepted tokens come as a step of their own
        pipeline.draft_step(by_hand.kv, by_hand.seqs, parents, rows, lambda out: paths, rotary, at)
        assert by_hand.seqs.lengths == s.seqs.lengths and by_hand.seqs.table == s.seqs.table
        batch, picked = by_hand.seqs.batch(n), [sum(len(p) for p in parents[:b]) + j for b, p in enumerate(paths) for j in p]
        for l in range(LAYERS):
            Q = rows(l)[0].clone()
            if rotary:
                other = binding.PagedKV(1, 4, H, D, store=store, page_tokens=PAGE)
                K = torch.zeros(Q.shape[0], H, D, device="cuda")
                table = torch.arange(1, dtype=torch.int32, device="cuda")[None]
                place = binding.PagedBatch(table, torch.tensor([Q.shape[0]], dtype=torch.int32, device="cuda"), torch.tensor([0, Q.shape[0]], dtype=torch.int32, device="cuda"),
                                           Q.shape[0], Q.shape[0], Q.shape[0])
                Q = other.scalekv_paged_write_rotated(0, place, Q, K, K, rotary, at)
            lse = torch.empty(sum(n), H * G, device="cuda")
            by_hand.kv.scalekv_paged_attend(l, batch, Q[picked], lse=lse)
            by_hand.kv.scalekv_paged_weigh(l, batch, Q[picked], lse, by_hand.weights[l], decay=0.9)
        for l in range(LAYERS):
            for b in range(3):
                got, want = s.sums(l, b), by_hand.sums(l, b)
                assert np.isfinite(got).all() and np.array_equal(got, want)
        keep = [40, 5, 20]
        before = [[s.sums(l, b) for b in range(3)] for l in range(LAYERS)]
        kept = pipeline.evict(s.kv, s.seqs, s.weights, keep, n_sink=1, n_recent=4)
        pipeline.evict(by_hand.kv, by_hand.seqs, by_hand.weights, keep, n_sink=1, n_recent=4)
        for l in range(LAYERS):
            for b in range(3):
                for h in range(H):
                    stay = po.stays(before[l][b][:, h], keep[b], 1, 4)
                    assert kept[l][b, h, :len(stay)].tolist() == stay.tolist()
                assert np.isfinite(s.sums(l, b)).all()
    s.kv.scalekv_paged_sync()
    by_hand.kv.scalekv_paged_sync()
