"""The codes that a write forms without divisions, against divisions: bf16 rows whose largest values and other values go through all significands, at scales
on both sides of the ones that are lifted and among the subnormal ones; f32 rows next to where codes change.  Codes and scales are compared bit for bit."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def held(c, n):
    """Codes [n, 1, d] and scales [n, 1] of K as they lie in the pool."""
    rows = c.kv.pool.numel() // (2 * (c.d + 4))
    codes = c.kv.pool[:rows * c.d].view(torch.int8).view(2, c.kv.n_pages, 1, c.page, c.d)
    scales = c.kv.pool[2 * rows * c.d:2 * rows * c.d + rows * 4].view(torch.float32).view(2, c.kv.n_pages, 1, c.page)
    pages = c.table[0, :-(-n // c.page)].long()
    return codes[c.layer, pages].reshape(-1, c.d)[:n].cpu().numpy(), scales[c.layer, pages].reshape(-1)[:n].cpu().numpy()


def check(x, dtype):
    """x [rows, d] float32, exact in dtype."""
    n, d = x.shape
    c = Case([1], [1], 1, d=d, page=128, spare=-(-n // 128))
    c.lengths = c.new = [n]
    c.table = torch.randperm(c.kv.n_pages, generator=torch.Generator().manual_seed(n)).to(torch.int32)[None].cuda()
    t = torch.from_numpy(x[:, None]).cuda().to(dtype)
    assert np.array_equal(t.float().cpu().numpy()[:, 0], x)
    c.kv.scalekv_paged_write(c.layer, c.batch(), t, t)
    c.kv.scalekv_paged_sync()
    codes, scales = held(c, n)
    want_codes, want_scales = po.quantise(x)
    assert np.array_equal(scales, want_scales)
    wrong = np.argwhere(codes != want_codes)
    assert len(wrong) == 0, [(float(x[r].max()), float(x[r, i]), int(codes[r, i]), int(want_codes[r, i])) for r, i in wrong[:5]]


def rows_of(largest, others, d):
    """Rows that begin with `largest` and hold all of `others`, signs in turn."""
    per = d - 1
    others = np.concatenate([others, np.zeros(-len(others) % per, np.float32)]).reshape(-1, per)
    others[:, ::2] *= -1
    return np.concatenate([np.full((len(others), 1), largest, np.float32), others], 1)


BF16 = np.float32(1) + np.arange(128, dtype=np.float32) / 128


# scales are lifted below 2^-60: largest values of about 2^-53
@pytest.mark.parametrize("exponent", [0, 127, 40, -52, -53, -54, -60, -100, -118, -126])
def test_bf16_rows_of_every_significand(exponent):
    others = np.concatenate([np.ldexp(BF16, exponent - k) for k in range(10)]).astype(np.float32)      # beyond 9 the code is 0
    others = np.unique(po.to_bf16(others))                                                             # (some are subnormal)
    x = np.concatenate([rows_of(a, others[others <= a], 128) for a in np.ldexp(BF16, exponent).astype(np.float32)])
    check(x.astype(np.float32), torch.bfloat16)


def test_bf16_rows_of_subnormal_values():
    unit = np.float32(2.0 ** -133)
    x = np.concatenate([rows_of(a, np.arange(1, n + 1, dtype=np.float32) * unit, 64) for n in range(1, 128) for a in [np.float32(n) * unit]])
    check(x, torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("low,high", [(-1, 1), (-126, 127), (-56, -50), (-140, -126)])
def test_f32_rows_where_codes_change(d, low, high):
    """Values at, next to and two places from (k + 1/2) s."""
    rng = np.random.default_rng(abs(d + high))
    n = 600
    a = np.ldexp(1 + rng.random(n), rng.integers(low, high + 1, n)).astype(np.float32)
    a = np.where(np.isfinite(a), a, np.float32(3e38))
    s = (a / np.float32(127)).astype(np.float32)
    k = np.stack([rng.permutation(127)[:d - 1] if d - 1 < 127 else np.arange(127) for _ in range(n)])
    at = (k + 0.5) * s[:, None].astype(np.float64)
    out = []
    for places in (-2, -1, 0, 1, 2):
        x = at.astype(np.float32)
        for _ in range(abs(places)):
            x = np.nextafter(x, np.float32(np.inf if places > 0 else 0))
        x = np.minimum(x, a[:, None])
        x[:, ::2] *= -1
        out.append(np.concatenate([a[:, None], x], 1))
    check(np.concatenate(out).astype(np.float32), torch.float32)
