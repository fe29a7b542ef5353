"""Whole numbers on their way through the native calls: a layer or a scale beyond 32 bits must not come out as another, valid one.  The library's functions
are stood in for by ones that note what they are given."""
import ctypes as C

import pytest

from paper_2505_19602_b200 import binding

torch = pytest.importorskip("torch")
T = binding.scalekv_tensor
LONG = [(2 ** 32 + 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (-2 ** 32 + 1, -2 ** 31), (2 ** 62, 2 ** 31 - 1), (1, 1), (-1, -1), (0, 0), (2 ** 31 - 1, 2 ** 31 - 1)]


def noting(*types):
    """A function of the library's kind, and the list of what it was called with."""
    seen = []

    def fn(*args):
        seen.append(args)
        return 0

    f = C.CFUNCTYPE(C.c_int, *types)(fn)
    return f, C.cast(f, C.c_void_p).value, seen


@pytest.mark.parametrize("given,want", LONG)
def test_layers_and_scales(given, want):
    call, x, i32, p = binding.load_call(), torch.zeros(1, 1, 2, 64), C.c_int32, C.c_void_p
    keep, fn, seen = noting(p, i32, i32, T, T)
    call.append(fn, 0, given, 3, x, x)
    call.append(fn, 0, 3, given, x, x)
    assert [s[1:3] for s in seen] == [(want, 3), (3, want)]
    keep, fn, seen = noting(p, i32, T, T, p)
    call.attend(fn, 0, given, x, x, None)
    assert seen[0][1] == want
    keep, fn, seen = noting(p, i32, T, i32, p, i32, p)
    call.compress_ex(fn, 0, given, x, given, 0, 0, 0)
    assert (seen[0][1], seen[0][3]) == (want, want)
    keep, fn, seen = noting(p, i32, i32, T, T, T, T, p, i32, p)
    call.step(fn, 0, given, given, x, x, x, x, None, given, 0)
    assert (seen[0][1], seen[0][2], seen[0][8]) == (want, want, want)


def test_no_number_at_all():
    call, x = binding.load_call(), torch.zeros(1, 1, 2, 64)
    keep, fn, seen = noting(C.c_void_p, C.c_int32, C.c_int32, T, T)
    for wrong, error in (("1", TypeError), (1.5, TypeError), (2 ** 64, OverflowError)):
        with pytest.raises(error):
            call.append(fn, 0, wrong, 0, x, x)
    assert not seen


@pytest.mark.gpu
def test_layers_of_the_paged_cache():
    from tests.test_paged_gpu import Case

    c = Case([20, 5], [1, 1], 2, 2, 64).fill()
    before = c.kv.pool.clone()
    new, Q = torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)
    for layer in (2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 31, -2 ** 31 - 1):
        for act in (lambda: c.kv.scalekv_paged_write(layer, c.batch(), new, new), lambda: c.kv.scalekv_paged_read(layer, c.batch()),
                    lambda: c.kv.scalekv_paged_attend(layer, c.batch(), Q)):
            with pytest.raises(binding.ScaleKVError, match="layer"):
                act()
    assert torch.equal(before, c.kv.pool)
    c.check()
