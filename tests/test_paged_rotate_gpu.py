"""Rows written with their positions in them against a plain implementation in 64 bits.

Tolerances.  A turned value a cos f - b sin f: the angle is off by 2^-22 and 2^-52 of itself (below 2^-21 for positions below 2^31 that turn by a radian at most), sine and
cosine by two units in their last place (2^-22 in all), and two products and a sum round by 2^-24 of |a| + |b| each: together below 2^-20 (|a| + |b|).  bf16 then rounds by 2^-8 of
the value.  Codes: half a scale, and the scale by 2^-24 of itself and what the row's largest value is off by / 127; a value of 127 codes is off by as much again."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def positions(rng, axes, n, far):
    p = rng.integers(-far, far, (axes, n), dtype=np.int64)
    p[:, :1] = 0
    return p.astype(np.int32)


def raw(c, name):
    """The pool's rows and scales of the case's layer: [page, head, row, d] numbers held, and scales."""
    rows = c.kv.pool.numel() // (2 * (c.d + 4) if c.store == "q8" else 4 * c.d)
    shape, i = (2, c.kv.n_pages, c.H, c.page), "KV".index(name)
    if c.store == "bf16":
        return c.kv.pool[i * rows * 2 * c.d:(i + 1) * rows * 2 * c.d].view(torch.bfloat16).view(*shape, c.d)[c.layer].float().cpu().numpy(), None
    codes = c.kv.pool[i * rows * c.d:(i + 1) * rows * c.d].view(torch.int8).view(*shape, c.d)[c.layer].cpu().numpy()
    at = 2 * rows * c.d + i * rows * 4
    return codes, c.kv.pool[at:at + rows * 4].view(torch.float32).view(shape)[c.layer].cpu().numpy()


def check(c, rotary, dtype, far=100000, Q=None, out=None, strides=None):
    T = sum(c.new)
    p = positions(c.rng, rotary.n_axes, T, far)
    x = [t.copy() for t in (c.Q, c.K[:T], c.V[:T])]
    if dtype == torch.bfloat16:
        x = [po.to_bf16(t) for t in x]
    Qd, K, V = (torch.from_numpy(t).cuda().to(dtype) for t in x)
    pd = torch.from_numpy(p).cuda()
    got = c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Qd, K, V, rotary, pd, Qd if out == "in place" else None)
    c.kv.scalekv_paged_sync()
    assert (got is Qd) == (out == "in place") and got.dtype == torch.bfloat16
    axis, freq = list(rotary.struct.axis)[:rotary.n_pairs], list(rotary.struct.frequency)[:rotary.n_pairs]
    want, A = po.turned(x[0], p, axis, freq, rotary.struct.adjacent)
    assert (np.abs(got.float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * A).all()
    want, A = po.turned(x[1], p, axis, freq, rotary.struct.adjacent)
    t, table = 0, c.table.cpu().numpy()
    (kr, ks), (vr, vs) = raw(c, "K"), raw(c, "V")
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        for i in range(n):
            pos = length - n + i
            at = table[b, pos // c.page], slice(None), pos % c.page
            if c.store == "bf16":
                assert (np.abs(kr[at] - want[t]) <= 2.0 ** -8 * np.abs(want[t]) + 2.0 ** -20 * A[t]).all()
                assert np.array_equal(vr[at], po.to_bf16(x[2][t]))
            else:
                s, top = ks[at].astype(np.float64), np.abs(want[t]).max(-1)
                off = 2.0 ** -20 * A[t].max(-1) / 127 + 2.0 ** -23 * s
                assert (np.abs(s - top / 127) <= off).all()
                assert (np.abs(kr[at] * s[:, None] - want[t]) <= (s / 2 + 127 * off)[:, None] + 2.0 ** -20 * A[t] + 2.0 ** -22 * np.abs(want[t])).all()
                codes, scales = po.quantise(x[2][t])
                assert np.array_equal(vr[at], codes) and np.array_equal(vs[at], scales)
            t += 1


ROTARIES = {64: [dict(sections=[32]), dict(sections=[8], adjacent=True), dict(sections=[5, 0, 19], in_turn=True), dict(sections=[10, 11, 11], own_range=True, adjacent=True)],
            128: [dict(sections=[16, 24, 24]), dict(sections=[64], adjacent=True, theta=1e6), dict(sections=[8, 8], own_range=True), dict(sections=[7, 7, 7, 35], in_turn=True, adjacent=True)]}


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("lengths,new,page,heads,group", [([1], [1], 16, 1, 1), ([40, 3, 0, 77], [2, 0, 0, 30], 16, 3, 2), ([200, 333], [200, 1], 64, 5, 4)])
def test_rotated_rows(store, dtype, d, which, lengths, new, page, heads, group):
    c = Case(lengths, new, heads, group, d, store, page, seed=which)
    check(c, binding.Rotary(**ROTARIES[d][which]), dtype)


def test_far_positions():
    for dtype in (torch.bfloat16, torch.float32):
        check(Case([300], [300], 2, 2, 128), binding.Rotary([32, 32]), dtype, far=2 ** 31 - 1)


def test_in_place_and_many_tokens():
    check(Case([3000, 9000], [3000, 7000], 1, 2, 64), binding.Rotary([32]), torch.bfloat16, out="in place")


def test_without_queries_and_strided_rows():
    c = Case([50, 21], [50, 21], 4, 2, 64)
    wide = torch.zeros(71, 3, 9, 72, device="cuda")
    Q, K, V = wide[:, 0, :8, :64], wide[:, 1, 1:5, :64], wide[:, 2, ::2, :64][:, 1:]
    for x, y in ((Q, c.Q), (K, c.K), (V, c.V)):
        x.copy_(torch.from_numpy(y).cuda())
    p = torch.from_numpy(positions(c.rng, 3, 71, 1000)).cuda()
    every = torch.zeros(3, 200, dtype=torch.int32, device="cuda")
    every[:, :71] = p
    r = binding.Rotary([8, 12, 12])
    out = torch.full((8, 71, 64), 5.0, device="cuda", dtype=torch.bfloat16)      # heads outermost
    c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q, K, V, r, every[:, :71], out.transpose(0, 1))
    pool = c.kv.pool.clone()
    dense = c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q.contiguous(), K.contiguous(), V.contiguous(), r, p)
    assert torch.equal(dense, out.transpose(0, 1)) and torch.equal(pool, c.kv.pool)
    c.kv.pool.fill_(255)
    assert c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), None, K, V, r, p) is None
    c.kv.scalekv_paged_sync()
    assert torch.equal(pool, c.kv.pool)


def test_position_zero_is_a_plain_write():
    c = Case([70], [70], 3, 1, 128)
    K, V = (torch.from_numpy(x).cuda() for x in (c.K, c.V))
    c.kv.scalekv_paged_write(c.layer, c.batch(), K, V)
    pool = c.kv.pool.clone()
    c.kv.pool.fill_(255)
    c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), None, K, V, binding.Rotary([64]), torch.zeros(1, 70, dtype=torch.int32, device="cuda"))
    c.kv.scalekv_paged_sync()
    assert torch.equal(pool, c.kv.pool)


def test_rows_that_are_no_numbers():
    c = Case([4], [4], 1, 1, 64)
    x = torch.ones(4, 1, 64, device="cuda")
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 63] = float("nan"), float("inf"), 0.0
    p = torch.tensor([[3, 4, 5, 6]], dtype=torch.int32, device="cuda")
    Q = c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), x, x, x, binding.Rotary([24]), p)
    K, V = c.kv.scalekv_paged_read(c.layer, c.batch(), dtype=torch.float32)
    assert torch.isnan(K[:2]).all() and torch.isnan(V[:2]).all() and torch.isfinite(K[2:]).all() and torch.isfinite(Q[2:]).all()
    assert torch.isnan(Q[0, 0, [3, 27]]).all() and int(torch.isfinite(Q[0]).sum()) == 62


def test_nothing_but_the_tokens_rows_changes():
    c = Case([40, 3, 77], [2, 0, 30], 3)
    before = c.kv.pool.clone()
    check(c, binding.Rotary([64]), torch.float32)
    rows = c.kv.pool.numel() // (2 * (c.d + 4))
    touched = torch.zeros(2, c.kv.n_pages, 3, 16, dtype=torch.bool)
    for b, (n, length) in enumerate(zip(c.new, c.lengths)):
        for pos in range(length - n, length):
            touched[1, int(c.table[b, pos // 16]), :, pos % 16] = True
    for part in torch.split((c.kv.pool != before).cpu(), [rows * c.d] * 2 + [rows * 4] * 2):
        assert not (part.view(*touched.shape, -1).any(-1) & ~touched).any()


def test_refusals():
    c = Case([40], [8], 2, 2, 64)
    K, V, Q = (torch.from_numpy(x[:8]).cuda() for x in (c.K, c.V, c.Q))
    p, r = torch.zeros(1, 8, dtype=torch.int32, device="cuda"), binding.Rotary([32])
    before = c.kv.pool.clone()
    for args in [(Q, K, V, r, p.float()), (Q, K, V, r, p[0]), (Q, K, V, r, p[:, :7]), (Q, K, V, binding.Rotary([16, 16]), p), (Q, K, V.bfloat16(), r, p),
                 (Q.bfloat16(), K, V, r, p), (Q, K, V, r, p.cpu()), (Q[:7], K, V, r, p), (Q, K, V, r, p, Q)]:
        with pytest.raises(ValueError):
            c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), *args)
    with pytest.raises(TypeError):
        c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q, K, None, r, p)
    wrong = binding.Rotary([64])
    with pytest.raises(binding.ScaleKVError, match="pairs"):
        c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q, K, V, wrong, p)
    r.struct.frequency[3] = float("inf")
    with pytest.raises(binding.ScaleKVError, match="frequency"):
        c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q, K, V, r, p)
    r.struct.frequency[3], r.struct.axis[5] = 1.0, 1
    with pytest.raises(binding.ScaleKVError, match="axis"):
        c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), Q, K, V, r, p)
    with pytest.raises(binding.ScaleKVError, match="layer"):
        c.kv.scalekv_paged_write_rotated(2, c.batch(), Q, K, V, binding.Rotary([32]), p)
    c.kv.scalekv_paged_sync()
    assert torch.equal(before, c.kv.pool)


def test_bad_pages_are_left_out_and_told():
    c = Case([40, 20], [40, 20], 2, 1, 64)
    before = c.kv.pool.clone()
    c.table[0, 1], c.table[1, 0] = c.kv.n_pages, -1
    K, V = (torch.from_numpy(x).cuda() for x in (c.K, c.V))
    p = torch.zeros(1, 60, dtype=torch.int32, device="cuda")
    c.kv.scalekv_paged_write_rotated(c.layer, c.batch(), None, K, V, binding.Rotary([32]), p)
    with pytest.raises(binding.ScaleKVError, match="DEVICE_CHECK"):
        c.kv.scalekv_paged_sync()
    rows = c.kv.pool.numel() // (2 * (c.d + 4))
    changed = (c.kv.pool != before)[:rows * c.d].view(2, c.kv.n_pages, 2, 16, 64).any(-1)
    assert int(changed[1, :, 0].sum()) == 24 + 4 and not changed[0].any()
