"""How far an exponent of the summed attention weights may be off."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from tests.test_paged_gpu import Case
from tests.test_paged_weigh_infinite_gpu import entries, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def weighed(c, lse, scale):
    """What each entry of the one sequence gets, [length, kv heads], in 32 bits and from the formula in 64."""
    w = torch.zeros(c.kv.n_pages, c.H, c.page, device="cuda")
    c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, w, causal=False, softmax_scale=scale)
    c.kv.scalekv_paged_sync()
    at, row = entries(c, 0)
    scale, n = float(np.float32(scale)), c.new[0]
    want, Y = np.zeros((c.lengths[0], c.H)), np.zeros((c.lengths[0], c.H))
    far = np.zeros((c.lengths[0], c.H))
    seen = np.ones((n, c.lengths[0]), bool)
    for h in range(c.H):
        k = c.rows(c.K, 0)[:, h]
        for g in range(h * c.G, (h + 1) * c.G):
            s, SY, SE = po.attention_got(c.Q[:, g], k, lse.cpu().numpy()[:, g], seen, scale)
            want[:, h] += s
            Y[:, h] += SY
            far[:, h] += SE
    return w[at, :, row].cpu().numpy().astype(np.float64), want, Y, far


@pytest.mark.parametrize("store", ["bf16", "q8"])
@pytest.mark.parametrize("new,group", [(1, 4), (1, 8), (4, 2), (8, 3)])
def test_far_exponents_of_few_rows_keep_their_last_bits(store, new, group):
    """Products that are exact (whole numbers, sums below 2^13), log-sum-exps and scaled products near 60.  In two floats an exponent E is off by 2 x 2^-24 of itself (one rounding of each part's
    sum), the exponential by 2^-22 of its result, the sum of n by n 2^-24.  (In one float the scaled log-sum-exp and the scaled product would be off by 2^-24 of 87 each, ten times that for the entries that count.)"""
    c = Case([64], [new], 1, group, 64, store)
    rng = np.random.default_rng(3)
    c.K[:] = rng.integers(-8, 9, c.K.shape)
    c.K[..., 0] = 127                                                 # (a scale of 1: codes are the numbers)
    c.Q[:] = rng.integers(-2, 3, c.Q.shape)
    c.Q[..., 0] = 4
    c.fill()
    scale = 60 / 508
    y = float(np.float32(scale)) * np.einsum("tgd,kd->tgk", c.Q.astype(np.float64), c.K[:, 0].astype(np.float64))
    lse = torch.from_numpy((y.max(-1) + rng.random(y.shape[:2])).astype(np.float32)).cuda()
    got, want, _, _ = weighed(c, lse, scale)
    exponent = np.abs(y - lse.cpu().numpy()[..., None])               # (natural: in base 2 log2 e times that, of which an error counts ln 2 times)
    tol = ((2.0 ** -22 + 2.0 ** -23 * exponent + new * group * 2.0 ** -24) * np.exp(-exponent)).sum((0, 1))[:, None]
    assert (np.abs(got - want) <= tol).all(), float(((got - want) / tol).max())


@pytest.mark.parametrize("store", ["bf16", "q8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,group", [(1, 4), (8, 4), (11, 3), (90, 1)])
def test_products_of_one_sign_and_a_key_that_dominates(store, d, new, group):
    """The bound that is stated for an exponent, tested where a sum's cut-offs all fall the same way: products of one sign, and a key several times as long as the others."""
    c = Case([96], [new], 2, group, d, store)
    c.K[:] = np.abs(c.K) * 0.2 + 0.01
    c.K[17] *= 6
    c.Q[:] = po.to_bf16(np.abs(c.Q) + 0.05)
    c.fill()
    scale = 16.0 / d
    lse = torch.from_numpy(np.stack([np.log(np.exp(scale * (c.Q[:, h].astype(np.float64) @ c.rows(c.K, 0)[:, h // group].T) - 30).sum(-1)) + 30
                                     for h in range(2 * group)], 1).astype(np.float32)).cuda()
    got, want, Y, far = weighed(c, lse, scale)
    few = new * group <= 32
    cut, itself = (2.0 ** -19, 2.0 ** -22) if few else (d * 2.0 ** -24, 2.0 ** -22)
    tol = cut * Y + itself * far + (new * group + 2) * 2.0 ** -24 * want
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
def test_products_that_lie_below_the_last_place(d, new):
    """A product of 1 and d - 1 of 1.5 x 2^-a, which a tensor core's sum loses one by one from some a on: the same bound.  (Of d - 1 products that are all lost, one sum over all dimensions would be
    off by 48 x 2^-24 at d = 128, above what is stated for few rows, and sums of 32 by 12.)"""
    c = Case([64], [new], 1, 1, d, "bf16")
    for j in range(64):
        c.K[j] = 1.5 * 2.0 ** -(14 + j // 4)
        c.K[j, 0, (0, d // 2, d - 1, 17)[j % 4]] = 1.0
    c.Q[:] = 1.0
    c.fill()
    lse = torch.full((new, 1), -float("inf"), device="cuda")
    lse[0] = 64.0
    got, want, Y, _ = weighed(c, lse, 64.0)
    # (in two floats an exponent is off by 2^-23 of itself; in one by the last places of 64 log2 e, twice)
    E = np.abs(Y / want - 64)
    tol = (2.0 ** -19 if new == 1 else d * 2.0 ** -24) * Y + (2.0 ** -22 + 2.0 ** -23 * E + (0 if new == 1 else 2 * 2.0 ** -24 * 64) + (new + 2) * 2.0 ** -24) * want
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
