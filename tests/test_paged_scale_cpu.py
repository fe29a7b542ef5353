"""A softmax_scale that 32 bits hold as 0, which stands for 1 / sqrt(head_dim), is refused by the native calls."""
import pytest

from paper_2505_19602_b200 import binding

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("scale", [1e-50, -1e-50, 5e-324, 7e-46])
def test_a_scale_that_is_lost_is_refused(scale):
    binding.build_library()
    call, x, f, i = binding.load_call(), torch.zeros(3, 2, 64).bfloat16(), torch.zeros(3, 2), torch.zeros(3, 1, dtype=torch.int32)
    w = torch.zeros(3, 2, 64)
    attend = lambda s: call.paged_attend(0, 0, 0, 0, 3, 64, 0, x, x, None, True, 0, 0, s, 0)  # noqa: E731
    tree = lambda s: call.paged_attend_tree(0, 0, 0, 0, 3, 64, 0, x, x, None, i, s, 0)  # noqa: E731
    weigh = lambda s: call.paged_weigh(0, 0, 0, 0, 3, 64, 0, x, f, w, 3, 2, 64, True, 0, 0, 1.0, s, 0)  # noqa: E731
    for act in (attend, tree, weigh):
        with pytest.raises(ValueError, match="softmax_scale"):
            act(scale)
        for held in (0.0, -0.0, 1e-45, 0.125):                        # (the next thing that is wrong: nothing here is on a device)
            with pytest.raises(ValueError, match="device"):
                act(held)
        with pytest.raises(TypeError):
            act(None)
