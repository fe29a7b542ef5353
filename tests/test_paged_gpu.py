"""The paged token cache against plain implementations: rows written and read back, and attention of single tokens and chunks.

Tolerances.  Written rows are compared exactly: the scale and the quotients are single fp32 operations.  O: the result is rounded to
bf16, whose unit roundoff is 2^-8 (8 significant bits), and so is every probability: 2^-8 of |O| and 2^-8 of A = sum p |v| at most; what fp32 sums and exponentials add is below 2^-12 of
A for the lengths here.  lse: an fp32 sum of d products and a scaling, 2 (d + 4) 2^-24 of Y = max sum |q k|, and 2^-18 of itself for
the exponentials, their sum and the logarithm."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Case:
    """Sequences with given lengths and numbers of new tokens in a pool that held NaN before, pages scattered, holes in the table."""

    def __init__(self, lengths, new, kv_heads, group=1, d=128, store="q8", page=16, layers=2, layer=1, seed=0, spare=2, wide=0):
        self.lengths, self.new, self.H, self.G, self.d, self.store, self.page, self.layer = lengths, new, kv_heads, group, d, store, page, layer
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-l // page) for l in lengths]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).astype(np.int32)
        table = np.full((len(lengths), max(need + [1]) + wide), -7, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = torch.from_numpy(table).cuda()
        self.kv = binding.PagedKV(layers, n_pages, kv_heads, d, store=store, page_tokens=page)
        self.kv.pool.fill_(255)                                   # codes of -1, scales and bf16 rows of NaN
        K = rng.standard_normal((sum(lengths), kv_heads, d)).astype(np.float32)
        K += 0.5 * rng.standard_normal((1, kv_heads, d)).astype(np.float32)
        K[::97] *= 4
        V = rng.standard_normal(K.shape).astype(np.float32)
        self.K, self.V = K, V
        self.Q = po.to_bf16(rng.standard_normal((sum(new), kv_heads * group, d)).astype(np.float32))

    def batch(self, new=None, lengths=None, max_length=None):
        new, lengths = self.new if new is None else new, self.lengths if lengths is None else lengths
        dev = dict(dtype=torch.int32, device="cuda")
        return binding.PagedBatch(self.table, torch.tensor(lengths, **dev), torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], **dev),
                                  sum(new), max(new + [1]), max(lengths) if max_length is None else max_length)

    def fill(self, dtype=torch.float32):
        self.kv.scalekv_paged_write(self.layer, self.batch(self.lengths), torch.from_numpy(self.K).cuda().to(dtype),
                                    torch.from_numpy(self.V).cuda().to(dtype))
        return self

    def rows(self, X, b):
        at = sum(self.lengths[:b])
        return po.stored(X[at:at + self.lengths[b]], self.store)

    def check(self, causal=True, window=0, n_sink=0, scale=0.0, Q=None, O=None, with_lse=True, max_length=None):
        T = sum(self.new)
        Qd = torch.from_numpy(self.Q).cuda().bfloat16() if Q is None else Q
        lse = torch.full((T, self.H * self.G), 7.0, device="cuda") if with_lse else None
        O = self.kv.scalekv_paged_attend(self.layer, self.batch(max_length=max_length), Qd, O, lse, causal, window, n_sink, scale)
        self.kv.scalekv_paged_sync()
        got, got_lse = O.float().cpu().numpy(), lse.cpu().numpy() if with_lse else None
        c = scale or 1 / math.sqrt(self.d)
        for b, (n, length) in enumerate(zip(self.new, self.lengths)):
            seen = po.visible(n, length, causal, window, n_sink)
            t0 = sum(self.new[:b])
            k, v = self.rows(self.K, b), self.rows(self.V, b)
            for h in range(self.H * self.G):
                want, want_lse, A, Y = po.attend(self.Q[t0:t0 + n, h], k[:, h // self.G], v[:, h // self.G], seen, c)
                err = np.abs(got[t0:t0 + n, h] - want)
                tol = 2.0 ** -8 * (np.abs(want) + A) + 2.0 ** -12 * A + 1e-30
                assert np.isfinite(got[t0:t0 + n, h]).all() and (err <= tol).all(), (b, h, float((err - tol).max()))
                if with_lse:
                    g = got_lse[t0:t0 + n, h]
                    empty = ~seen.any(1)
                    assert (g[empty] == -np.inf).all() and (got[t0:t0 + n, h][empty] == 0).all()
                    tol = 2 * (self.d + 4) * 2.0 ** -24 * Y + 2.0 ** -18 * (1 + np.abs(want_lse))
                    assert (np.abs(g[~empty] - want_lse[~empty]) <= tol[~empty]).all(), (b, h)


# ---- rows written and read back --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths,page,heads", [([1], 16, 1), ([17, 0, 1, 64, 5], 16, 3), ([100, 333, 16], 64, 5), ([130] * 9, 128, 2)])
def test_rows_come_back_as_they_are_held(store, d, dtype, lengths, page, heads):
    c = Case(lengths, lengths, heads, d=d, store=store, page=page)
    K, V = (torch.from_numpy(x).cuda().to(dtype) for x in (c.K, c.V))
    c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
    got = c.kv.scalekv_paged_read(c.layer, c.batch(), dtype=torch.float32) + c.kv.scalekv_paged_read(c.layer, c.batch(), dtype=torch.bfloat16)
    c.kv.scalekv_paged_sync()
    for i, x in enumerate((K, V, K, V)):
        want = po.stored(x.float().cpu().numpy(), store)
        assert np.array_equal(got[i].float().cpu().numpy(), want if i < 2 else po.to_bf16(want))


def test_rows_of_the_layer_and_of_the_tokens_alone_change():
    c = Case([40, 3, 77], [2, 0, 30], 3)
    before = c.kv.pool.clone()
    K, V = (torch.from_numpy(x[:32]).cuda() for x in (c.K, c.V))
    c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
    c.kv.scalekv_paged_sync()
    rows = c.kv.pool.numel() // (2 * (c.d + 4))
    shape = (2, c.kv.n_pages, 3, 16)
    touched = torch.zeros(shape, dtype=torch.bool)
    table = c.table.cpu()
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        for pos in range(length - n, length):
            touched[1, table[b, pos // 16], :, pos % 16] = True
    for i, part in enumerate(torch.split((c.kv.pool != before).cpu(), [rows * c.d] * 2 + [rows * 4] * 2)):
        changed = part.view(*shape, -1).any(-1)
        assert not (changed & ~touched).any() and bool(changed[touched].float().mean() > 0.99), i


def test_rows_that_are_no_numbers_and_rows_of_nothing():
    c = Case([6], [6], 1, d=64)
    x = np.zeros((6, 1, 64), np.float32)
    x[0, 0, 3], x[1, 0, 63], x[2, 0, 0] = np.nan, np.inf, -np.inf
    x[4], x[5, 0, 5] = 1e-45, 3e38
    t = torch.from_numpy(x).cuda()
    c.kv.scalekv_paged_write(c.layer, c.batch(), t, t)
    K, V = c.kv.scalekv_paged_read(c.layer, c.batch(), dtype=torch.float32)
    for got in (K.cpu().numpy(), V.cpu().numpy()):
        assert np.isnan(got[:3]).all() and (got[3:5] == 0).all()
        assert np.array_equal(got[5], po.stored(x[5], "q8"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_rows(dtype):
    c = Case([50, 21], [50, 21], 4, d=64)
    wide = torch.zeros(71, 3, 6, 72, device="cuda", dtype=dtype)
    K, V = wide[:, 0, 1:5, :64], wide[:, 2, ::1, :64][:, 2:]
    K.copy_(torch.from_numpy(c.K).cuda())
    V.copy_(torch.from_numpy(c.V).cuda())
    c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
    out = torch.full((2, 4, 71, 64), 5.0, device="cuda", dtype=dtype)      # heads outermost
    c.kv.scalekv_paged_read(c.layer, c.batch(), out[0].transpose(0, 1), out[1].transpose(0, 1))
    for got, x in zip(out, (K, V)):
        want = po.stored(x.float().cpu().numpy(), "q8")
        want = want if dtype == torch.float32 else po.to_bf16(want)
        assert np.array_equal(got.transpose(0, 1).float().cpu().numpy(), want)


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off", [(16, 16), (0, 16), (16, 0)])
def test_rows_that_begin_on_16_bytes(dtype, store, off):
    """K, V or both begin on 16 bytes but not on 32, in as in out; the same rows are held and come back."""
    c = Case([50, 21], [50, 21], 4, d=64, store=store)
    esize = torch.empty(0, dtype=dtype).element_size()
    flat = [torch.zeros(71 * 4 * 64 + 16, device="cuda", dtype=dtype) for _ in range(4)]
    K, V, K_out, V_out = (f[o // esize:][: 71 * 4 * 64].view(71, 4, 64) for f, o in zip(flat, off + off))
    assert [x.data_ptr() % 32 for x in (K, V)] == list(off)
    K.copy_(torch.from_numpy(c.K).cuda())
    V.copy_(torch.from_numpy(c.V).cuda())
    c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
    c.kv.scalekv_paged_read(c.layer, c.batch(), K_out, V_out)
    for got, x in zip((K_out, V_out), (K, V)):
        want = po.stored(x.float().cpu().numpy(), store)
        want = want if dtype == torch.float32 else po.to_bf16(want)
        assert np.array_equal(got.float().cpu().numpy(), want)
    assert all(bool((f[o // esize + 71 * 4 * 64:] == 0).all()) and bool((f[: o // esize] == 0).all()) for f, o in zip(flat, off + off))


# ---- attention -------------------------------------------------------------------------------------------------------------------
LENGTHS = [1, 2, 15, 16, 17, 31, 128, 129, 300]


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (2, 4), (1, 16), (2, 7), (1, 40)])
def test_single_tokens(store, d, kv_heads, group):
    Case(LENGTHS, [1] * len(LENGTHS), kv_heads, group, d, store).fill().check()


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 128), ("q8", 64), ("bf16", 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,new,group", [([37], [37], 1), ([5, 200, 130, 64], [3, 0, 130, 9], 2), ([700, 260], [257, 129], 1),
                                               ([300, 299, 1], [150, 1, 1], 5), ([1000], [33], 8)])
def test_chunks(store, d, causal, lengths, new, group):
    Case(lengths, new, 2, group, d, store, page=32).fill().check(causal)


@pytest.mark.parametrize("store,d", [("q8", 128), ("bf16", 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (7, 3), (16, 16), (100, 4), (128, 130), (5000, 2), (33, 300)])
def test_windows_and_sinks(store, d, causal, window, n_sink):
    lengths = [1, 18, 500, 333, 129]
    Case(lengths, [1] * 5, 2, 3, d, store).fill().check(causal, window, n_sink)
    Case(lengths, [1, 18, 200, 1, 0], 2, 3, d, store).fill().check(causal, window, n_sink)


@pytest.mark.parametrize("group", [1, 8])
def test_queries_of_a_cache_that_does_not_hold_them(group):
    """Queries beside the sequence: lengths below the number of new tokens, down to nothing; where the mask is causal such rows are
    empty."""
    for causal in (True, False):
        Case([0, 5, 40, 0], [3, 9, 41, 1], 2, group).fill().check(causal)
        Case([0, 5, 40, 0], [3, 9, 200, 1], 2, group, store="bf16").fill().check(causal, window=6, n_sink=2)


@pytest.mark.parametrize("store", ["q8", "bf16"])
def test_many_keys_shared_by_several_ctas(store):
    Case([5003], [1], 1, 4, 128, store, page=64).fill().check()
    Case([5003, 70], [2, 1], 1, 4, 64, store, page=64).fill().check(window=3000, n_sink=9)
    Case([3001], [40], 1, 2, 128, store, page=64).fill().check()
    Case([3001, 2], [300, 2], 1, 1, 128, store, page=64).fill().check()


@pytest.mark.parametrize("max_length", [0, 1, 100000])
def test_the_longest_length_only_sizes_the_launch(max_length):
    Case([700, 31], [1, 1], 2, 2).fill().check(max_length=max_length)
    Case([700, 31], [200, 31], 2, 2).fill().check(max_length=max_length)


def test_large_products_and_a_scale():
    for new in ([1, 1], [150, 90]):
        c = Case([200, 90], new, 1, 2)
        c.Q = po.to_bf16(c.Q * 30)
        c.fill().check(scale=0.5)                  # products of several hundred: all but one key of a row vanish
        c.check(scale=0.001, with_lse=False)


def test_references_that_rise_late():
    """Keys whose products grow with the position: the running maximum rises again and again, far into the sequence."""
    for store in ("q8", "bf16"):
        for new in (1, 130):
            c = Case([900], [new], 1, 1, 128, store)
            c.K *= np.linspace(0.05, 6, 900, dtype=np.float32)[:, None, None]
            c.K[-1] *= 2
            c.Q = np.abs(c.Q)
            c.K = np.abs(c.K)
            c.fill().check(causal=False)


def test_strided_queries_and_outputs():
    for new in ([1, 1, 1], [20, 150, 1]):
        c = Case([64, 150, 7], new, 2, 3, 64).fill()
        T = sum(new)
        wide = torch.full((T, 3, 8, 80), 9.0, device="cuda", dtype=torch.bfloat16)
        Q, O = wide[:, 0, 1:7, 8:72], wide[:, 1, 2:, :64]
        Q.copy_(torch.from_numpy(c.Q).cuda())
        kept = wide.clone()
        c.check(Q=Q, O=O)
        kept[:, 1, 2:, :64] = O
        assert torch.equal(kept, wide)


@pytest.mark.parametrize("new", [[1, 1], [140, 1]])
def test_hidden_rows_may_hold_anything(new):
    """Keys that a mask hides from some rows or from all: NaN rows (NaN scales) ahead of the window, behind a causal query, and pages
    of the window's past that have been given back (table entries of nonsense)."""
    c = Case([400, 300], new, 2, 2, 128, "q8").fill()
    for b, length in enumerate(c.lengths):
        hidden = max(0, length - new[b] - 50)
        at = sum(c.lengths[:b])
        bad = np.zeros(c.K.shape[0], bool)
        bad[at + 20:at + hidden] = True
        c.K[bad], c.V[bad] = np.nan, np.inf
    c.fill()
    c.K[~np.isfinite(c.K)], c.V[~np.isfinite(c.V)] = 0, 0           # (for the oracle, which multiplies what it hides)
    for b, length in enumerate(c.lengths):
        c.table[b, 2:(length - new[b] - 50) // 16] = 123456
    c.check(window=50, n_sink=20)


def test_a_row_that_is_no_number_reaches_those_that_see_it_and_nobody_else():
    for store in ("q8", "bf16"):
        c = Case([200], [200], 1, 1, 128, store).fill()
        K = torch.from_numpy(c.K).cuda()
        V = torch.from_numpy(c.V).cuda()
        K[150, 0, 5] = float("nan")
        if store == "q8":
            V[170, 0, 3] = float("inf")
        c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
        lse = torch.empty(200, 1, device="cuda")
        O = c.kv.scalekv_paged_attend(c.layer, c.batch(), torch.from_numpy(c.Q).cuda().bfloat16(), lse=lse)
        assert torch.isfinite(O[:150]).all() and torch.isfinite(lse[:150]).all()
        assert torch.isnan(O[150:]).all() and torch.isnan(lse[150:]).all()


def test_the_same_twice_and_on_other_streams():
    c = Case([2000, 700, 90], [1, 1, 1], 2, 4, 128, page=64).fill()
    Q = torch.from_numpy(c.Q).cuda().bfloat16()
    torch.cuda.synchronize()
    first = c.kv.scalekv_paged_attend(c.layer, c.batch(), Q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        batch = c.batch()
        for _ in range(3):
            again = c.kv.scalekv_paged_attend(c.layer, batch, Q)
        c.kv.scalekv_paged_sync()
    assert torch.equal(first, again)


def test_a_captured_step_replays():
    """Write and attend captured once; the lengths move on the device between replays."""
    c = Case([60, 33], [1, 1], 2, 2, 128, "q8", spare=6, wide=2)
    c.fill()
    free = [p for p in range(c.kv.n_pages) if p not in set(c.table.flatten().tolist())]
    for b, length in enumerate(c.lengths):
        for i in range(2):
            c.table[b, -(-length // 16) + i] = free[2 * b + i]
    batch = c.batch(max_length=100)
    rng = np.random.default_rng(1)
    K, V, Q = (torch.zeros(2, h, 128, device="cuda", dtype=torch.bfloat16) for h in (2, 2, 4))
    O = torch.zeros_like(Q)

    def step():
        c.kv.scalekv_paged_write(c.layer, batch, K, V)
        c.kv.scalekv_paged_attend(c.layer, batch, Q, O)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(20):
        batch.tensors[1].add_(1)
        for x in (K, V, Q):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)))
        graph.replay()
        got = O.clone()
        step()
        assert torch.equal(got, O)
        at = np.cumsum([0] + c.lengths)
        c.K, c.V = (np.concatenate([np.concatenate([X[at[b]:at[b + 1]], x[b:b + 1].float().cpu().numpy()]) for b in (0, 1)])
                    for X, x in ((c.K, K), (c.V, V)))
        c.lengths = [l + 1 for l in c.lengths]
    c.Q = Q.float().cpu().numpy()
    c.check()


def test_offsets_beyond_32_bits():
    """A pool whose rows lie more than 2^32 bytes apart: the last pages of the last layer."""
    kv = binding.PagedKV(3, 20000, 4, 128, store="bf16", page_tokens=128)
    assert kv.pool.numel() > 3 * 2 ** 32
    c = Case([300, 129], [1, 1], 4, 2, 128, "bf16", page=128)
    c.kv, c.layer = kv, 2
    c.table.copy_(torch.tensor([[19999, 19996, 19990], [0, 19998, -1]]))
    c.fill().check()
    c.new = [70, 129]
    c.Q = po.to_bf16(np.random.default_rng(3).standard_normal((199, 8, 128)).astype(np.float32))
    c.check()


# ---- refusals --------------------------------------------------------------------------------------------------------------------
def test_refusals():
    c = Case([20, 5], [1, 1], 2, 2, 64).fill()
    good = torch.zeros(2, 2, 64, device="cuda")
    Q = torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)
    for K in (good[:1], good[:, :1], good[..., :32], good.half(), good.cpu(), good.transpose(1, 2), torch.zeros(2, 2, 128, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_write(c.layer, c.batch(), K, good)
    with pytest.raises(ValueError):
        c.kv.scalekv_paged_write(c.layer, c.batch(), good, good.bfloat16())
    with pytest.raises(TypeError):
        c.kv.scalekv_paged_write(c.layer, c.batch(), None, good)
    for layer in (-1, 2):
        with pytest.raises(binding.ScaleKVError, match="layer"):
            c.kv.scalekv_paged_read(layer, c.batch())
    for wrong in (Q.float(), Q[:, :3], Q[:1]):
        with pytest.raises((ValueError, binding.ScaleKVError)):
            c.kv.scalekv_paged_attend(c.layer, c.batch(), wrong)
    for kw in ({"window": -1}, {"n_sink": -3}, {"softmax_scale": float("nan")}, {"softmax_scale": -1.0}, {"lse": torch.zeros(2, 3, device="cuda")},
               {"lse": torch.zeros(2, 4, device="cuda", dtype=torch.bfloat16)}, {"O": Q[:, :2]}):
        with pytest.raises((ValueError, binding.ScaleKVError)):
            c.kv.scalekv_paged_attend(c.layer, c.batch(), Q, **kw)
    odd = torch.zeros(2 * 4 * 64 + 8, device="cuda", dtype=torch.bfloat16)[1:513].view(2, 4, 64)
    with pytest.raises(binding.ScaleKVError, match="aligned"):
        c.kv.scalekv_paged_attend(c.layer, c.batch(), odd)
    i32 = dict(dtype=torch.int32, device="cuda")
    for args in ((c.table.long(), torch.zeros(2, **i32), torch.zeros(3, **i32), 0, 1, 1), (c.table, torch.zeros(3, **i32), torch.zeros(4, **i32), 0, 1, 1),
                 (c.table, torch.zeros(2, **i32), torch.zeros(2, **i32), 0, 1, 1), (c.table.cpu(), torch.zeros(2, **i32), torch.zeros(3, **i32), 0, 1, 1),
                 (c.table, torch.zeros(2, **i32), torch.zeros(3, **i32), -1, 1, 1)):
        with pytest.raises(ValueError):
            binding.PagedBatch(*args)
    with pytest.raises(binding.ScaleKVError):
        binding.PagedKV(1, 1, 1, 96)
    with pytest.raises(binding.ScaleKVError):
        binding.PagedKV(1, 1, 1, 64, page_tokens=24)
    with pytest.raises(binding.ScaleKVError):
        binding.PagedKV(1, 4, 1, 64, pool=torch.zeros(100, dtype=torch.uint8, device="cuda"))
    c.check()


def test_no_tokens_and_no_sequences():
    c = Case([20, 5], [0, 0], 2).fill()
    none = torch.zeros(0, 2, 128, device="cuda", dtype=torch.bfloat16)
    launches = c.kv.scalekv_paged_launch_count()
    c.kv.scalekv_paged_write(c.layer, c.batch(), none, none)
    assert c.kv.scalekv_paged_attend(c.layer, c.batch(), none).shape == (0, 2, 128)
    i32 = dict(dtype=torch.int32, device="cuda")
    empty = binding.PagedBatch(torch.zeros(0, 4, **i32), torch.zeros(0, **i32), torch.zeros(1, **i32), 0, 0, 0)
    c.kv.scalekv_paged_read(c.layer, empty)
    assert c.kv.scalekv_paged_launch_count() == launches
    c.kv.scalekv_paged_sync()


def test_pages_and_lengths_out_of_range_are_reported_and_left_out():
    def fresh():
        return Case([100, 40], [1, 1], 2, 2).fill()

    c = fresh()
    c.table[0, 3], c.table[1, 1] = 10 ** 6, -1
    before = c.kv.pool.clone()
    K, V = c.kv.scalekv_paged_read(c.layer, c.batch([100, 40]), dtype=torch.float32)
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()
    assert (K[48:64] == 0).all() and (K[116:132] == 0).all() and np.array_equal(K[:48].cpu().numpy(), po.stored(c.K[:48], "q8"))
    c.kv.scalekv_paged_write(c.layer, c.batch([60, 20]), torch.ones(80, 2, 128, device="cuda"), torch.ones(80, 2, 128, device="cuda"))
    torch.cuda.synchronize()
    assert not torch.equal(before, c.kv.pool)
    # attention: the keys of a page that is out of range count as hidden
    for new in (1, 90):
        c = fresh()
        c.new = [new, 1]
        c.Q = po.to_bf16(c.rng.standard_normal((new + 1, 4, 128)).astype(np.float32))
        c.table[0, 3] = 10 ** 6
        O = c.kv.scalekv_paged_attend(c.layer, c.batch(), torch.from_numpy(c.Q).cuda().bfloat16()).float().cpu().numpy()
        with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
            c.kv.scalekv_paged_sync()
        seen = po.visible(new, 100, True, 0, 0)
        seen[:, 48:64] = False
        for h in range(4):
            want, _, A, _ = po.attend(c.Q[:new, h], c.rows(c.K, 0)[:, h // 2], c.rows(c.V, 0)[:, h // 2], seen, 128 ** -0.5)
            assert (np.abs(O[:new, h] - want) <= 2.0 ** -8 * (np.abs(want) + A) + 2.0 ** -12 * A).all()
    # a length beyond the table, more new tokens than promised, tokens of no sequence
    for lengths, starts, tokens in (([5000, 40], [0, 1, 2], 2), ([100, 40], [0, 1, 9], 9), ([100, 40], [0, 1, 2], 6), ([100, 40], [5, 1, 2], 6)):
        c = fresh()
        i32 = dict(dtype=torch.int32, device="cuda")
        batch = binding.PagedBatch(c.table, torch.tensor(lengths, **i32), torch.tensor(starts, **i32), tokens, 2, 5000)
        c.kv.scalekv_paged_read(c.layer, batch)
        c.kv.scalekv_paged_attend(c.layer, batch, torch.zeros(tokens, 4, 128, device="cuda", dtype=torch.bfloat16))
        with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
            c.kv.scalekv_paged_sync()
