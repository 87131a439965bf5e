"""CPU tests of numbers that a call's arguments hold and the C entry points' 32-bit fields do
not: they are refused, not cut.  The tensors are of no memory and call themselves the
device's; nothing is launched."""
import pytest

torch = pytest.importorskip("torch")

from paper_2304_00338_amd import mgn  # noqa: E402


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def rows(r, c, dtype=torch.bfloat16):
    return torch.empty(r, c, dtype=dtype, device="meta").as_subclass(OnDevice)


@pytest.mark.parametrize("cols,groups", [((1 << 32) + 128, 32), ((1 << 32) + 128, 1), (64, (1 << 32) + 4), (64, 4 - (1 << 32)),
                                         (64, 0), (64, -4), (64, 128), (16385, 5), (0, 1)])
def test_group_norm_columns_and_groups(cols, groups):
    x = rows(1, cols)
    stats = torch.empty(1, 4, 2, device="meta").as_subclass(OnDevice)
    for call in (lambda: mgn.mgn_group_norm_forward(x, groups), lambda: mgn.mgn_group_norm_backward(x, stats, x, groups)):
        with pytest.raises(mgn.MgnError) as e:
            call()
        assert e.value.code in (mgn.ERR_ARG, mgn.ERR_SHAPE)
