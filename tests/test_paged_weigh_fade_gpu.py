"""Sums of entries that a window hides: left alone, or faded like the others."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding, pipeline
from tests.test_paged_gpu import Case
from tests.test_paged_weigh_infinite_gpu import queries, sums

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,causal", [([1, 1, 0, 2], True), ([70, 3, 0, 40], True), ([5, 9, 0, 1], False)])
@pytest.mark.parametrize("window,n_sink", [(50, 0), (33, 7), (1, 16), (64, 200), (9999, 3)])
def test_hidden_entries_fade_where_they_are_asked_to(new, causal, window, n_sink):
    """All entries before the new tokens fade, hidden ones by one product; the others' sums are those of a call that leaves hidden ones alone."""
    lengths = [400, 90, 200, 333]
    c = Case(lengths, new, 2, 2, 64).fill()
    lse, old = torch.full((sum(new), 4), 4.0, device="cuda"), sums(c)
    if not po.visible(new[0], 400, causal, window, n_sink).any(0)[32:48].any():
        c.table[0, 2] = -1                                            # (a page that was given back is passed over)
    for max_length in (None, 1):
        alone, w = old.clone(), old.clone()
        c.kv.scalekv_paged_weigh(c.layer, c.batch(max_length=max_length), queries(c), lse, alone, causal, window, n_sink, 0.75)
        c.kv.scalekv_paged_weigh(c.layer, c.batch(max_length=max_length), queries(c), lse, w, causal, window, n_sink, 0.75, fade_hidden=True)
        c.kv.scalekv_paged_sync()
        want = alone.clone()
        for b, (n, length) in enumerate(zip(new, lengths)):
            hidden = ~po.visible(n, length, causal, window, n_sink).any(0) if n else np.zeros(length, bool)
            assert not hidden[length - n:].any()
            pos = np.flatnonzero(hidden)
            page = c.table.cpu().numpy()[b, pos // c.page]
            pos, page = pos[page >= 0], page[page >= 0]
            p, r = torch.from_numpy(page).cuda().long(), torch.from_numpy(pos % c.page).cuda()
            assert torch.equal(alone[p, :, r], old[p, :, r])
            want[p, :, r] = old[p, :, r] * 0.75
        assert torch.equal(w, want)


def test_nothing_fades_without_a_window_or_a_decay():
    c = Case([200], [2], 1, 1, 64).fill()
    lse, old = torch.full((2, 1), 4.0, device="cuda"), sums(c)
    for kw in ({"decay": 0.5}, {"window": 20}):
        a, b = old.clone(), old.clone()
        launches = c.kv.scalekv_paged_launch_count()
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, a, **kw)
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, b, fade_hidden=True, **kw)
        assert torch.equal(a, b) and c.kv.scalekv_paged_launch_count() == launches + 2
    c.kv.scalekv_paged_sync()


def test_refused_fades():
    c = Case([100], [4], 2, 2, 64).fill()
    w = sums(c)
    old = w.clone()
    for args, error, what in (((w, -1, 0, 0.5), ValueError, "window"), ((w, 5, 2 ** 31, 0.5), ValueError, "n_sink"), ((w[1:], 5, 0, 0.5), ValueError, "weights"),
                              ((w.half(), 5, 0, 0.5), ValueError, "weights"), ((w, 5, 0, 1.5), binding.ScaleKVError, "decay"),
                              ((w, 5, 0, float("nan")), binding.ScaleKVError, "decay"),
                              ((torch.zeros(w.numel() + 1, device="cuda")[1:].view(w.shape), 5, 0, 0.5), binding.ScaleKVError, "aligned")):
        with pytest.raises(error, match=what):
            c.kv.scalekv_paged_fade(c.layer, c.batch(), *args)
    with pytest.raises(binding.ScaleKVError, match="layer"):
        c.kv.scalekv_paged_fade(7, c.batch(), w, 5, 0, 0.5)
    c.kv.scalekv_paged_sync()
    assert torch.equal(w, old)


def test_fades_are_captured_and_tell_of_lengths_out_of_range():
    c = Case([400], [2], 2, 1, 64).fill()
    old = sums(c)
    w, batch = old.clone(), c.batch()
    c.kv.scalekv_paged_fade(c.layer, batch, w, 50, 5, 0.5)
    want = w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.kv.scalekv_paged_fade(c.layer, batch, w, 50, 5, 0.5)
    w.copy_(old)
    graph.replay()
    c.kv.scalekv_paged_sync()
    assert torch.equal(w, want) and not torch.equal(w, old)
    c.kv.scalekv_paged_fade(c.layer, c.batch(lengths=[1 << 20]), w, 50, 5, 0.5)
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()


def test_sums_under_a_window_fade_alike():
    """An entry that a window hides ranks by the same fading as one that it shows; one whose page was given back leaves the page's next owner alone."""
    rng = np.random.default_rng(5)
    kv, seqs, weights = binding.PagedKV(2, 20, 2, 64, page_tokens=16), pipeline.Sequences(20, 16, 1, 200), torch.full((2, 20, 2, 16), float("nan"), device="cuda")

    def held(l):
        pos = np.arange(seqs.lengths[0])
        return weights[l].cpu().numpy()[np.array(seqs.table[0])[pos // 16], :, pos % 16]

    def step(n):
        seqs.extend([n])
        given = [[torch.from_numpy(rng.standard_normal((n, h, 64)).astype(np.float32)).cuda().bfloat16() for h in (4, 2, 2)] for _ in range(2)]
        pipeline.token_step(kv, seqs.batch([n]), lambda l: given[l], window=20, n_sink=2, weights=weights, decay=0.5)

    step(90)
    before = [held(l) for l in range(2)]
    step(1)
    for l in range(2):
        got = held(l)
        assert np.array_equal(got[2:71], before[l][2:71] * np.float32(0.5)) and (got[71:90] > 0.5 * before[l][71:]).all()
    seqs.trim(20, 2)
    assert seqs.table[0][1:4] == [-1] * 3 and seqs.table[0][4] >= 0
    old = weights.clone()
    step(1)
    pages = [p for p in seqs.table[0] if p >= 0]
    gone = [p for p in range(20) if p not in pages]
    assert torch.equal(weights[:, gone].view(torch.int32), old[:, gone].view(torch.int32)) and not torch.equal(weights[:, pages], old[:, pages])
    kv.scalekv_paged_sync()
