"""The paged token cache as a program drives it: prompts in chunks beside single tokens over several layers, pages given back behind a
window; and cases drawn over the ranges of sizes, masks and stores.  Tolerances as derived in test_paged_gpu.py."""
import math
import random

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding, pipeline
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store,d,window,n_sink", [("q8", 128, 0, 0), ("q8", 64, 40, 5), ("bf16", 128, 33, 0)])
def test_prompts_and_tokens(store, d, window, n_sink):
    prompts, n_tokens, H, G, layers = [70, 1, 0, 130, 33], 6, 2, 3, 3
    rng = np.random.default_rng(7)
    total = [p + n_tokens for p in prompts]
    data = [[tuple(po.to_bf16(rng.standard_normal((n, h, d)).astype(np.float32)) for h in (H * G, H, H)) for n in total] for _ in range(layers)]
    pages = sum(-(-n // 16) for n in total) + 1 if not window else 5 * (window + n_sink + 64 + 48) // 16
    kv = binding.PagedKV(layers, pages, H, d, store=store, page_tokens=16)
    kv.pool.fill_(255)
    seqs = pipeline.Sequences(pages, 16, len(prompts), max(total))

    def rows(layer, counts, positions):
        return tuple(torch.from_numpy(np.concatenate([data[layer][b][i][p:p + n] for b, (n, p) in enumerate(zip(counts, positions))])).cuda().bfloat16()
                     for i in range(3))

    got = [[np.zeros((n, H * G, d), np.float32) for n in total] for _ in range(layers)]
    for counts, positions, out in pipeline.prompts_and_tokens(kv, seqs, prompts, n_tokens, 64, rows, window, n_sink):
        for l, O in enumerate(out):
            at = 0
            for b, (n, p) in enumerate(zip(counts, positions)):
                got[l][b][p:p + n] = O[at:at + n].float().cpu().numpy()
                at += n
    kv.scalekv_paged_sync()
    assert seqs.lengths == total
    for l in range(layers):
        for b, n in enumerate(total):
            Q, K, V = data[l][b]
            seen = po.visible(n, n, True, window, n_sink)
            for h in range(H * G):
                want, _, A, _ = po.attend(Q[:, h], po.stored(K, store)[:, h // G], po.stored(V, store)[:, h // G], seen, d ** -0.5)
                assert (np.abs(got[l][b][:, h] - want) <= 2.0 ** -8 * (np.abs(want) + A) + 2.0 ** -12 * A).all(), (l, b, h)
    for b in range(len(prompts)):
        seqs.drop(b)
    assert sorted(seqs.free) == list(range(pages))


@pytest.mark.parametrize("seed", range(40))
def test_drawn_cases(seed):
    r = random.Random(seed)
    n = r.choice([1, 1, 2, 5, 9, 40])
    d, store, page = r.choice([64, 128]), r.choice(["q8", "bf16"]), r.choice([16, 32, 64, 128])
    kv_heads, group = r.choice([1, 2, 3, 5]), r.choice([1, 1, 2, 4, 7, 8, 16])
    longest = r.choice([20, 150, 700, 2500]) if n < 9 else r.choice([20, 150, 400])
    new = r.choice([[1] * n, [r.choice([0, 1, 2]) for _ in range(n)], [r.randint(0, min(longest, 300)) for _ in range(n)]])
    if not any(new):
        new[0] = 1
    causal = r.random() < 0.7
    lengths = [max(r.randint(0, longest), k if r.random() < 0.8 else 0) for k in new]
    window = r.choice([0, 0, r.randint(1, 300)])
    c = Case(lengths, new, kv_heads, group, d, store, page, seed=seed)
    c.Q = po.to_bf16(c.Q * r.choice([0.3, 1.0, 4.0]))
    c.fill()
    c.check(causal, window, r.choice([0, 1, 17]) if window else 0)


@pytest.mark.parametrize("lengths,heads", [([2000, 900, 1500, 30, 1999, 1200, 77], 8), ([1500] * 12, 8), ([3000, 5], 16), ([64] * 300, 4)])
def test_many_sequences_of_different_lengths(lengths, heads):
    """Launches whose parts are dealt out by the lengths; all rows against a plain fp32 attention on the GPU."""
    for store, group in (("q8", 4), ("bf16", 1)):
        c = Case(lengths, [1] * len(lengths), heads, group, 128, store, page=64).fill()
        lse = torch.empty(len(lengths), heads * group, device="cuda")
        Q = torch.from_numpy(c.Q).cuda().bfloat16()
        O = c.kv.scalekv_paged_attend(c.layer, c.batch(), Q, lse=lse).float()
        again = c.kv.scalekv_paged_attend(c.layer, c.batch(), Q).float()
        c.kv.scalekv_paged_sync()
        assert torch.equal(O, again)
        for b, length in enumerate(lengths):
            k, v = (torch.from_numpy(c.rows(x, b)).cuda().double().repeat_interleave(group, 1) for x in (c.K, c.V))
            y = torch.einsum("hd,lhd->hl", Q[b].double(), k) / math.sqrt(128)
            p = torch.softmax(y, -1)
            want, A = torch.einsum("hl,lhd->hd", p, v), torch.einsum("hl,lhd->hd", p, v.abs())
            assert bool(((O[b] - want).abs() <= 2.0 ** -8 * (want.abs() + A) + 2.0 ** -12 * A).all()), b
            Y = torch.einsum("hd,lhd->hl", Q[b].double().abs(), k.abs()).amax(-1) / math.sqrt(128)
            want_lse = torch.logsumexp(y, -1)
            assert bool(((lse[b] - want_lse).abs() <= 2 * 132 * 2.0 ** -24 * Y + 2.0 ** -18 * (1 + want_lse.abs())).all()), b


@pytest.mark.parametrize("lengths,new,heads", [([4200], [600], 1), ([3300, 3200], [1000, 200], 24), ([2000] * 3, [256] * 3, 60), ([900], [40], 5)])
def test_items_shared_by_several_ctas(lengths, new, heads):
    """Chunks whose last wave of items, or all of them, are shared; against fp64 on the GPU."""
    for store, d in (("q8", 64), ("bf16", 128)):
        c = Case(lengths, new, heads, 1, d, store, page=128).fill()
        Q = torch.from_numpy(c.Q).cuda().bfloat16()
        lse = torch.empty(sum(new), heads, device="cuda")
        O = c.kv.scalekv_paged_attend(c.layer, c.batch(), Q, lse=lse).double()
        c.kv.scalekv_paged_sync()
        at = 0
        for b, (n, length) in enumerate(zip(new, lengths)):
            k, v = (torch.from_numpy(c.rows(x, b)).cuda().double() for x in (c.K, c.V))
            seen = torch.from_numpy(po.visible(n, length, True, 0, 0)).cuda()
            y = torch.einsum("nhd,lhd->hnl", Q[at:at + n].double(), k) / math.sqrt(d)
            y.masked_fill_(~seen, -math.inf)
            p = torch.softmax(y, -1)
            want, A = torch.einsum("hnl,lhd->nhd", p, v), torch.einsum("hnl,lhd->nhd", p, v.abs())
            assert bool(((O[at:at + n] - want).abs() <= 2.0 ** -8 * (want.abs() + A) + 2.0 ** -12 * A).all()), b
            assert bool(((lse[at:at + n].T - torch.logsumexp(y, -1)).abs() <= 2.0 ** -13).all()), b
            at += n
