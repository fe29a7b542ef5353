"""Summed attention weights of keys that hold infinities and NaN: what the formula says, and nobody else's sum."""
import numpy as np
import pytest

from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def queries(c):
    return torch.from_numpy(c.Q).cuda().bfloat16()


def sums(c, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(c.kv.n_pages, c.H, c.page, generator=g, device="cuda") * 3 + 0.1


def entries(c, b):
    """Pages and rows of all positions of sequence b."""
    pos = np.arange(c.lengths[b])
    return torch.from_numpy(c.table.cpu().numpy()[b, pos // c.page]).cuda().long(), torch.from_numpy(pos % c.page).cuda()


@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (1, 8), (3, 5), (31, 1), (40, 1), (90, 3)])
@pytest.mark.parametrize("what,pays", [(-np.inf, 0.0), (np.inf, np.inf), (np.nan, np.nan)])
def test_an_infinite_key_pays_what_the_formula_says(new, group, what, pays):
    """Rows whose products with a key are all -inf pay it exp(-inf) = 0, those of +inf infinity, NaN NaN; nobody else's sum changes by a bit."""
    c = Case([300], [new], 2, group, 64, "bf16")
    c.Q[..., 3] = np.abs(c.Q[..., 3]) + 0.5
    lse, old = torch.full((new, 2 * group), 4.0, device="cuda"), sums(c)
    got = []
    at, row = entries(c, 0)
    for value in (1.0, what):
        for p in (0, 77, 160, 255):
            c.K[p, 1, 3] = value
        c.fill()
        w = old.clone()
        c.kv.scalekv_paged_weigh(c.layer, c.batch(), queries(c), lse, w, decay=0.5)
        got.append(w[at, :, row])
    c.kv.scalekv_paged_sync()
    was, faded = got[0].clone(), (0.5 * old[at, :, row])
    for p in (0, 77, 160, 255):
        first = 300 - new                                             # (of a new one nothing is left of what was there)
        was[p, 1] = (faded[p, 1] if p < first else 0.0) + pays
    assert torch.equal(was.isnan(), got[1].isnan()) and torch.equal(was.nan_to_num(7.0), got[1].nan_to_num(7.0))
