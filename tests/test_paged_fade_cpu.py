"""Fading without a GPU: refusals of the library and of the native call."""
import pytest

from paper_2505_19602_b200 import binding

torch = pytest.importorskip("torch")


def test_refused_fades():
    binding.build_library()
    assert binding.load_library().scalekv_paged_fade(None, 0, None, None, None, 1.0, None) == 1
    call, w = binding.load_call(), torch.zeros(3, 2, 64)
    for act, error, what in [(lambda: call.paged_fade(0, 0), TypeError, "arguments"),
                             (lambda: call.paged_fade(0, 0, 0, 0, 0, w, 3, 2, 64, -1, 0, 1.0, 0), ValueError, "window"),
                             (lambda: call.paged_fade(0, 0, 0, 0, 0, w, 3, 2, 64, 1, 2 ** 31, 1.0, 0), ValueError, "n_sink"),
                             (lambda: call.paged_fade(0, 0, 0, 0, 0, w, 4, 2, 64, 1, 0, 1.0, 0), ValueError, "weights"),
                             (lambda: call.paged_fade(0, 0, 0, 0, 0, w, 3, 2, 64, 1, 0, 1.0, 0), ValueError, "device"),
                             (lambda: call.paged_fade(0, 0, 0, 0, 0, None, 3, 2, 64, 1, 0, 1.0, 0), TypeError, "weights")]:
        with pytest.raises(error, match=what):
            act()
