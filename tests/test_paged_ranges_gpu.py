"""Values and keys of unusual size in the paged cache: what the header promises of them."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from tests.test_paged_gpu import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1], [12, 3, 1], [150, 90, 1]])
@pytest.mark.parametrize("exponent", [100, -100])
def test_large_and_small_values(store, d, new, exponent):
    c = Case([700, 90, 1], new, 2, 2, d, store)
    c.V = np.ldexp(c.V, exponent).astype(np.float32)
    c.Q = po.to_bf16(c.Q * 3)
    c.fill().check()


@pytest.mark.parametrize("store", ["q8", "bf16"])
@pytest.mark.parametrize("new", [[1, 1], [12, 3], [150, 90]])
@pytest.mark.parametrize("exponent", [60, -60])
def test_large_and_small_keys(store, new, exponent):
    """Products of the usual size from keys and queries of any."""
    c = Case([700, 90], new, 2, 2, 128, store)
    c.K, c.Q = np.ldexp(c.K, exponent).astype(np.float32), po.to_bf16(np.ldexp(c.Q, -exponent).astype(np.float32))
    c.fill().check()
