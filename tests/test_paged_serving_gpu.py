"""Rotated writes, drafts, summed weights and eviction as a server uses them: one behind the other, captured and replayed, on a stream of their own.

Tolerances as in test_paged_gpu.py (O) and test_paged_rotate_gpu.py: rows are compared as the cache holds them, so what attention reads is the same on both sides."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding, pipeline

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
LAYERS, H, G, D, PAGE = 2, 2, 2, 64, 16
ROTARY = binding.Rotary([8, 12, 12])


def draw(rng, n, heads):
    return rng.standard_normal((n, heads, D)).astype(np.float32)


class Server:
    """The cache and, beside it, every sequence's rows as the cache gives them back: what they hold is checked when they are written."""

    def __init__(self, n_seqs, store, seed=0):
        self.rng = np.random.default_rng(seed)
        self.kv = binding.PagedKV(LAYERS, 120, H, D, store=store, page_tokens=PAGE)
        self.kv.pool.fill_(255)
        self.seqs = pipeline.Sequences(120, PAGE, n_seqs, 600)
        self.weights = torch.full((LAYERS, 120, H, PAGE), float("nan"), device="cuda")
        self.rows = [[[np.zeros((0, H, D)) for _ in range(2)] for _ in range(n_seqs)] for _ in range(LAYERS)]
        self.q = {}

    def bring(self, new):
        """New tokens' Q, K, V for every layer, and their positions."""
        T = sum(new)
        self.new, self.given = new, [[draw(self.rng, T, n) for n in (H * G, H, H)] for _ in range(LAYERS)]
        self.positions = torch.from_numpy(self.rng.integers(0, 50000, (3, T)).astype(np.int32)).cuda()
        return lambda l: [torch.from_numpy(x).cuda() for x in self.given[l]]

    def queries(self, l):
        f = list(ROTARY.struct.frequency)[:32]
        return po.turned(self.given[l][0], self.positions.cpu().numpy(), list(ROTARY.struct.axis)[:32], f, 0)[0]

    def read(self, l, b, length):
        """What the cache holds of a sequence, as numbers."""
        table = torch.tensor([self.seqs.table[b]], dtype=torch.int32, device="cuda")
        batch = binding.PagedBatch(table, torch.tensor([length], dtype=torch.int32, device="cuda"), torch.tensor([0, length], dtype=torch.int32, device="cuda"), length, length, length)
        return [x.cpu().numpy() for x in self.kv.scalekv_paged_read(l, batch, dtype=torch.float32)]

    def check(self, out, before, sees=None):
        """Every layer's outputs, over rows that are what was there before and the new ones, turned and quantised."""
        f, axis, pos = list(ROTARY.struct.frequency)[:32], list(ROTARY.struct.axis)[:32], self.positions.cpu().numpy()
        for l in range(LAYERS):
            Q, got = self.queries(l), out[l].float().cpu().numpy()
            K, A = po.turned(self.given[l][1], pos, axis, f, 0)
            for b, n in enumerate(self.new):
                if n == 0:
                    continue
                t0 = sum(self.new[:b])
                k, v = self.read(l, b, before[b] + n)
                for x, old in zip((k, v), self.rows[l][b]):
                    assert np.array_equal(x[:before[b]], old)
                step = np.abs(K[t0:t0 + n]).max(-1, keepdims=True) / 127 if self.kv.store == "q8" else 2.0 ** -7 * np.abs(K[t0:t0 + n])
                assert (np.abs(k[before[b]:] - K[t0:t0 + n]) <= 0.51 * step + 2.0 ** -19 * A[t0:t0 + n]).all()
                assert np.array_equal(v[before[b]:], po.stored(self.given[l][2][t0:t0 + n], self.kv.store))
                seen = po.visible(n, before[b] + n, True, 0, 0) if sees is None else po.draft_visible(sees[b], before[b] + n)
                for h in range(H * G):
                    q = Q[t0:t0 + n, h]
                    want, _, S, Y = po.attend(q, k[:, h // G], v[:, h // G], seen, 1 / math.sqrt(D))
                    # (the queries went out as bf16: a product is off by 2^-8 of Y, a p by as much of itself, and O by twice that of sum p |v|)
                    tol = 2.0 ** -8 * (np.abs(want) + S) + 2.0 ** -12 * S + 2 * 2.0 ** -8 * Y[:, None] * S + 1e-30
                    assert (np.abs(got[t0:t0 + n, h] - want) <= tol).all()
                self.rows[l][b] = [k, v]


@pytest.mark.parametrize("store", ["q8", "bf16"])
def test_prompts_drafts_and_evictions_one_behind_the_other(store):
    s = Server(3, store)
    rng = s.rng
    for turn in range(3):
        for new in ([130, 7, 60], [1, 1, 1], [40, 0, 1]):                   # prompts and chunks, tokens one by one
            before = list(s.seqs.lengths)
            rows = s.bring(new)
            s.seqs.extend(new)
            out = pipeline.token_step(s.kv, s.seqs.batch(new), rows, rotary=ROTARY, positions=s.positions, weights=s.weights, decay=0.9)
            s.check(out, before)
        before = list(s.seqs.lengths)
        parents = [[int(rng.integers(-1, i)) if i else -1 for i in range(n)] for n in (20, 5, 3 * turn)]
        rows = s.bring([len(p) for p in parents])
        paths = [sorted(rng.choice(len(p), min(len(p), 3), replace=False).tolist()) for p in parents]

        def accept(out):
            sees = []
            for p in parents:
                seen = []
                for i, j in enumerate(p):
                    seen.append((seen[j] if j >= 0 else []) + [i])
                sees.append(seen)
            s.check(out, before, sees)
            return paths

        _, got = pipeline.draft_step(s.kv, s.seqs, parents, rows, accept, ROTARY, s.positions)
        assert got == paths and s.seqs.lengths == [a + len(p) for a, p in zip(before, paths)]
        for l in range(LAYERS):
            for b, p in enumerate(paths):
                s.rows[l][b] = [np.concatenate([x[:before[b]], x[before[b]:][p]]) for x in s.rows[l][b]]
        # the accepted tokens get their weights: their queries, and the attention that they paid as if they had come one by one
        counts = [len(p) for p in paths]
        at = [sum(s.new[:b]) + j for b, p in enumerate(paths) for j in p]
        batch = s.seqs.batch(counts)
        for l in range(LAYERS):
            Q = torch.from_numpy(po.to_bf16(s.queries(l)[at].astype(np.float32))).cuda().bfloat16()
            lse = torch.empty(len(at), H * G, device="cuda")
            s.kv.scalekv_paged_attend(l, batch, Q, lse=lse)
            s.kv.scalekv_paged_weigh(l, batch, Q, lse, s.weights[l], decay=0.9)
        keep = [50, 5, 1000]
        old, lengths, weights = [row[:] for row in s.seqs.table], list(s.seqs.lengths), s.weights.cpu().numpy()
        kept = pipeline.evict(s.kv, s.seqs, s.weights, keep, n_sink=2, n_recent=10)
        assert s.seqs.lengths == [min(k, x) for k, x in zip(keep, lengths)]
        for l in range(LAYERS):
            got = kept[l].cpu().numpy()
            for b, length in enumerate(lengths):
                pos = np.arange(length)
                page = np.array(old[b])[pos // PAGE]
                stay = []
                for h in range(H):
                    w = weights[l, page, h, pos % PAGE]
                    assert np.isfinite(w).all() and (w >= 0).all()
                    stay.append(po.stays(w, keep[b], 2, 10))
                    assert got[b, h, :len(stay[h])].tolist() == stay[h].tolist()
                s.rows[l][b] = [np.stack([x[stay[h], h] for h in range(H)], 1) for x in s.rows[l][b]]
                for x, want in zip(s.read(l, b, s.seqs.lengths[b]), s.rows[l][b]):
                    assert np.array_equal(x, want)
    s.kv.scalekv_paged_sync()
    held = [p for row in s.seqs.table for p in row if p >= 0]
    assert sorted(s.seqs.free + held) == list(range(120))


class Step:
    """Tensors of one serving step, all calls in it; they can be filled anew."""

    def __init__(self, kv, new, pages, layer=0, kv_seed=0):
        self.kv, self.layer, T, B = kv, layer, sum(new), len(new)
        dev = dict(dtype=torch.int32, device="cuda")
        self.new, self.table = new, torch.full((B, pages), -1, **dev)
        self.lengths, self.starts = torch.zeros(B, **dev), torch.tensor([sum(new[:b]) for b in range(B + 1)], **dev)
        self.batch = binding.PagedBatch(self.table, self.lengths, self.starts, T, max(new), 16 * pages)
        self.Q, self.K, self.V = (torch.zeros(T, n, D, device="cuda") for n in (H * G, H, H))
        self.positions, self.tree = torch.zeros(3, T, **dev), torch.zeros(T, -(-max(new) // 32), **dev)
        self.path, self.counts = torch.zeros(B, 4, **dev), torch.zeros(B, **dev)
        self.to, self.keep = torch.zeros(B, 2, **dev), torch.zeros(B, **dev)
        self.q, self.O = (torch.zeros(T, H * G, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.lse, self.weights = torch.zeros(T, H * G, device="cuda"), torch.zeros(kv.n_pages, H, PAGE, device="cuda")
        self.kept = torch.zeros(B, H, 32, **dev)

    def fill(self, seed):
        rng = np.random.default_rng(seed)
        B, pages = self.table.shape
        order = rng.permutation(self.kv.n_pages).astype(np.int32)
        put = lambda t, x: t.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(t.dtype))  # noqa: E731
        put(self.table, order[:B * pages].reshape(B, pages))
        put(self.to, order[B * pages:B * (pages + 2)].reshape(B, 2))
        put(self.lengths, rng.integers(max(self.new) + 40, 16 * pages + 1, B))
        for t in (self.Q, self.K, self.V):
            put(t, rng.standard_normal(tuple(t.shape)))
        put(self.positions, rng.integers(0, 9999, tuple(self.positions.shape)))
        tree = rng.integers(-2 ** 31, 2 ** 31, tuple(self.tree.shape))
        put(self.tree, tree)
        counts = rng.integers(0, 5, B)
        put(self.counts, counts)
        put(self.path, np.sort(np.stack([rng.choice(min(n, 9), 4, replace=False) for n in self.new]), 1))
        put(self.keep, rng.integers(1, 33, B))
        put(self.weights, rng.random(tuple(self.weights.shape)))
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = torch.randint(0, 100, self.kv.pool.shape, generator=g, device="cuda", dtype=torch.uint8)      # (finite as codes, scales or bf16)
        self.kv.pool.copy_(rows)
        for t in (self.q, self.O, self.lse, self.kept):
            t.zero_()

    def run(self):
        kv, l, b = self.kv, self.layer, self.batch
        kv.scalekv_paged_write_rotated(l, b, self.Q, self.K, self.V, ROTARY, self.positions, self.q)
        kv.scalekv_paged_attend_tree(l, b, self.q, self.tree, self.O, self.lse)
        kv.scalekv_paged_weigh(l, b, self.q, self.lse, self.weights, decay=0.5)
        kv.scalekv_paged_accept(b, self.path, self.counts)
        kv.scalekv_paged_evict(l, b, self.to, self.keep, self.weights, 2, 5, self.kept)

    def results(self):
        return [x.clone() for x in (self.q, self.O, self.lse, self.weights, self.kept, self.kv.pool)]


def same(a, b):
    return all(torch.equal(x.reshape(-1).view(torch.uint8), y.reshape(-1).view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("new", [[6, 5, 7], [40, 60, 9]])
def test_a_captured_step_follows_what_its_tensors_hold(store, new):
    kv = binding.PagedKV(2, 80, H, D, store=store, page_tokens=PAGE)
    s = Step(kv, new, 20)
    want = []
    for seed in (1, 2, 3):
        s.fill(seed)
        s.run()
        kv.scalekv_paged_sync()
        want.append(s.results())
    graph = torch.cuda.CUDAGraph()
    s.fill(4)
    with torch.cuda.graph(graph):
        s.run()
    for seed in (1, 2, 3, 1):
        s.fill(seed)
        graph.replay()
        kv.scalekv_paged_sync()
        assert same(s.results(), want[seed - 1]), seed


def test_steps_on_streams_of_their_own():
    """Two caches, two streams, nothing between them; results are those of one behind the other."""
    caches = [binding.PagedKV(2, 80, H, D, store="q8", page_tokens=PAGE) for _ in range(2)]
    steps, want = [Step(kv, new, 20) for kv, new in zip(caches, ([6, 5, 7], [40, 60, 9]))], []
    for i, s in enumerate(steps):
        s.fill(i)
        s.run()
        s.kv.scalekv_paged_sync()
        want.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for i, s in enumerate(steps):
            s.fill(i)
        torch.cuda.synchronize()
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.run()
        torch.cuda.synchronize()
        assert all(same(s.results(), w) for s, w in zip(steps, want))
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.kv.scalekv_paged_sync()


def everything(kv, first_page, heads, d, new=40, length=200, strided=False, seed=0):
    """All calls once on one sequence whose pages begin at first_page; what comes out, and what the cache then holds."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = dict(dtype=torch.int32, device="cuda")
    pages = -(-length // kv.page_tokens)
    table = torch.arange(first_page, first_page + pages, **dev)[None]
    to = torch.arange(first_page + pages, first_page + 2 * pages, **dev)[None]
    random = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    weights = torch.zeros(kv.n_pages, heads, kv.page_tokens, device="cuda")

    def batch(n):
        return binding.PagedBatch(table, torch.tensor([length], **dev), torch.tensor([0, n], **dev), n, n, length)

    def rows(n, h):
        x = random(n, h, d).bfloat16()
        if not strided:
            return x
        wide = torch.zeros(h + 3, n, 2, d + 8, device="cuda", dtype=x.dtype)      # heads outermost, odd steps
        wide[:h, :, 1, :d] = x.transpose(0, 1)
        return wide[:h, :, 1, :d].transpose(0, 1)

    r, out = binding.Rotary([d // 4, d // 4]), []
    position = torch.randint(0, 10000, (2, length), generator=g, **dev)
    kv.scalekv_paged_write_rotated(0, batch(length), None, rows(length, heads), rows(length, heads), r, position)
    for n in (1, new):
        bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, 2), generator=g, **dev)
        q = kv.scalekv_paged_write_rotated(0, batch(n), rows(n, 2 * heads), rows(n, heads), rows(n, heads), r, position[:, :n])
        lse = torch.empty(n, 2 * heads, device="cuda")
        out += [q, kv.scalekv_paged_attend_tree(0, batch(n), rows(n, 2 * heads), bits, lse=lse), lse.clone()]
        Q = rows(n, 2 * heads)
        kv.scalekv_paged_attend(0, batch(n), Q, lse=lse)
        kv.scalekv_paged_weigh(0, batch(n), Q, lse, weights, decay=0.5)
    kv.scalekv_paged_accept(batch(new), torch.tensor([[1, 5, 30]], **dev), torch.tensor([3], **dev))
    out += [kv.scalekv_paged_evict(0, batch(0), to, torch.tensor([100], **dev), weights, 3, 7)[:, :, :100], weights[first_page:first_page + 2 * pages]]
    out += list(kv.scalekv_paged_read(0, batch(length), dtype=torch.float32))
    kept = binding.PagedBatch(to, torch.tensor([100], **dev), torch.tensor([0, 100], **dev), 100, 100, 100)
    out += list(kv.scalekv_paged_read(0, kept, dtype=torch.float32))
    kv.scalekv_paged_sync()
    return out


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 64)])
def test_strides_change_nothing(store, d):
    kv = binding.PagedKV(1, 40, 3, d, store=store, page_tokens=16)
    kv.pool.zero_()
    assert same([x.contiguous() for x in everything(kv, 4, 3, d)], [x.contiguous() for x in everything(kv, 4, 3, d, strided=True)])


@pytest.mark.parametrize("store", ["q8", "bf16"])
def test_offsets_beyond_32_bits(store):
    """The same in a small pool and behind the first 4 GB of K rows of a large one."""
    small = binding.PagedKV(1, 12, 16, 128, store=store, page_tokens=64)
    pages = 36000 if store == "q8" else 18000                            # 4.7 GB of K rows
    large = binding.PagedKV(1, pages, 16, 128, store=store, page_tokens=64)
    for kv in (small, large):
        kv.pool.zero_()
    assert same(*([x.contiguous() for x in everything(kv, first, 16, 128)] for kv, first in ((small, 2), (large, pages - 9))))
