"""The paged token cache without a GPU: sizes and refusals of the C ABI, the sequences' page book, the oracle's own rules."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2505_19602_b200 import binding, pipeline


@pytest.fixture(scope="module")
def lib():
    binding.build_library()
    return binding.load_library()


def config(n_layers=2, n_pages=10, page_tokens=64, n_kv_heads=4, head_dim=128, store=1):
    return binding.scalekv_paged_config(n_layers, n_pages, page_tokens, n_kv_heads, head_dim, store)


def sizes(lib, cfg):
    pb, wb = C.c_size_t(0), C.c_size_t(0)
    return lib.scalekv_paged_query_sizes(C.byref(cfg), C.byref(pb), C.byref(wb)), pb.value, wb.value


def test_sizes(lib):
    rows = 2 * 10 * 64 * 4
    assert sizes(lib, config())[:2] == (0, 2 * rows * (128 + 4))
    assert sizes(lib, config(store=0))[:2] == (0, 2 * rows * 128 * 2)
    assert sizes(lib, config(head_dim=64))[:2] == (0, 2 * rows * (64 + 4))
    assert 0 < sizes(lib, config())[2] < 64 << 20


@pytest.mark.parametrize("wrong,status", [({"n_layers": 0}, "INVALID_ARG"), ({"n_pages": 0}, "INVALID_ARG"), ({"n_kv_heads": -1}, "INVALID_ARG"),
                                          ({"page_tokens": 8}, "INVALID_ARG"), ({"page_tokens": 48}, "INVALID_ARG"), ({"head_dim": 96}, "UNSUPPORTED"),
                                          ({"store": 7}, "INVALID_ARG"), ({"n_pages": 2 ** 26}, "CAPACITY")])
def test_refused_configurations(lib, wrong, status):
    assert binding.STATUS_NAMES[sizes(lib, config(**wrong))[0]] == status


def test_null_arguments(lib):
    assert lib.scalekv_paged_query_sizes(None, None, None) == 1
    assert lib.scalekv_paged_init(None, None) == 1
    out = C.c_void_p(1)
    assert lib.scalekv_paged_init(C.byref(config()), C.byref(out)) == 1 and not out.value          # no pool
    rows = binding.scalekv_rows(None, 0, 0)
    assert lib.scalekv_paged_write(None, 0, None, rows, rows, 0, None) == 1
    assert lib.scalekv_paged_read(None, 0, None, rows, rows, 0, None) == 1
    assert lib.scalekv_paged_attend(None, 0, None, 1, rows, rows, None, None, 0.0, None) == 1
    assert lib.scalekv_paged_sync(None, None) == 1 and lib.scalekv_paged_destroy(None) == 1
    assert lib.scalekv_paged_launch_count(None, None) == 1 and lib.scalekv_paged_error_string(None)


def test_no_cpu_path():
    import torch

    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(RuntimeError):
        binding.PagedKV(1, 1, 1, 64)
    t = torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.PagedBatch(t, t[0, :1], torch.zeros(2, dtype=torch.int32), 0, 1, 1)


def test_native_module_refuses_tensors_that_are_not_on_the_device():
    import torch

    call = binding.load_call()
    x = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError, match="device"):
        call.paged_move(0, 0, 0, 0, 3, 2, 64, 0, x, x, 0)
    with pytest.raises(ValueError, match="shape"):
        call.paged_move(0, 0, 0, 0, 4, 2, 64, 0, x, x, 0)
    with pytest.raises(TypeError):
        call.paged_attend(0, 0, 0, 0, 3, 64, 0, None, x, None, True, 0, 0, 0.0, 0)
    with pytest.raises(TypeError):
        call.paged_attend(0, 0)
    with pytest.raises(ValueError, match="window"):
        call.paged_attend(0, 0, 0, 0, 3, 64, 0, x, x, None, True, -1, 0, 0.0, 0)


def test_page_book():
    s = pipeline.Sequences(10, 16, 3, 100)
    s.extend([17, 0, 16])
    assert s.lengths == [17, 0, 16] and len(s.free) == 7
    s.extend([15, 1, 1])
    assert len(s.free) == 5 and sorted(p for row in s.table for p in row if p >= 0) == sorted(set(range(10)) - set(s.free))
    with pytest.raises(MemoryError):
        s.extend([0, 60, 60])
    with pytest.raises(ValueError):
        s.extend([100, 0, 0])
    assert s.lengths == [32, 1, 17] and len(s.free) == 5                    # refusals change nothing
    s.extend([48, 0, 0])                                                    # 80 entries: 5 pages
    s.trim(window=20, n_sink=3)                                             # the next token, at 80, sees [61, 80] and [0, 3)
    assert [p >= 0 for p in s.table[0][:5]] == [True, False, False, True, True] and len(s.free) == 4
    s.extend([5, 0, 0])
    assert s.table[0][1] == -1 and s.table[0][5] >= 0
    for b in range(3):
        s.drop(b)
    assert sorted(s.free) == list(range(10)) and s.lengths == [0, 0, 0]


def test_oracle_rows():
    x = np.array([[1.0, -127.0, 0.5, 63.5], [0, 0, 0, 0], [np.nan, 1, 2, 3], [1, np.inf, 0, 0], [2.5, 1.5, -0.5, 127]], np.float32)
    codes, s = po.quantise(x)
    assert codes[0].tolist() == [1, -127, 0, 64] and s[0] == 1            # halves go to the even code
    assert codes[1].tolist() == [0] * 4 and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3]) and not codes[2:4].any()
    assert codes[4].tolist() == [2, 2, 0, 127]
    assert po.to_bf16(np.float32([1.00390625, 1.01171875])).tolist() == [1.0, 1.015625]
    seen = po.visible(3, 8, True, 2, 1)
    assert seen.astype(int).tolist() == [[1, 0, 0, 0, 1, 1, 0, 0], [1, 0, 0, 0, 0, 1, 1, 0], [1, 0, 0, 0, 0, 0, 1, 1]]
    assert not po.visible(4, 2, True, 0, 0)[:2].any()                      # queries ahead of the sequence


def test_oracle_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((2, 4)), rng.standard_normal((5, 4)), rng.standard_normal((5, 4))
    seen = np.array([[True] * 5, [False] * 5])
    O, lse, A, Y = po.attend(q, k, v, seen, 0.5)
    e = np.exp(0.5 * k @ q[0])
    assert np.allclose(O[0], e @ v / e.sum()) and np.isclose(lse[0], np.log(e.sum())) and (A >= np.abs(O) - 1e-12).all() and Y[0] >= np.abs(0.5 * k @ q[0]).max()
    assert not O[1].any() and lse[1] == -np.inf
