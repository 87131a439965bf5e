"""CPU tests of what the binding says of matrices of one row, whose row stride means nothing but
whose columns have to be adjacent all the same.  The tensors are of host memory that
calls itself the device's; nothing is launched."""
import pytest

torch = pytest.importorskip("torch")

from paper_2304_00338_amd import mgn  # noqa: E402


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def on(t):
    return t.as_subclass(OnDevice)


def spread(rows, dtype):
    """Rows of 32 elements that are not adjacent: every second one of 64, a column of a
    matrix of 32 rows, and one element for all."""
    wide = torch.zeros(rows, 64, dtype=dtype)
    tall = torch.zeros(32, 3, dtype=dtype)
    return [wide[:, ::2], tall[:, :1].t(), torch.zeros(1, 1, dtype=dtype).expand(rows, 32)]


def scale4(rows, cols):
    return torch.zeros(-(-cols // 128), rows, 4, dtype=torch.uint8)


@pytest.mark.parametrize("rows", [1, 2])
def test_mat4_columns_apart(rows):
    for q in spread(rows, torch.uint8):
        if q.shape[0] == rows:
            for cols in (64, 33):
                with pytest.raises(mgn.MgnError, match="adjacent"):
                    mgn.Mat4(on(q), scale4(rows, cols), cols)


def test_mat4_one_row_of_any_stride():
    """A row inside a wider matrix, one of an odd number of bytes, and none."""
    wide = on(torch.zeros(5, 75, dtype=torch.uint8))
    for q, cols, ld in ((wide[2:3, 16:48], 60, 32), (wide[:1], 96, 80), (wide[:1, :16], 32, 16)):
        m = mgn.Mat4(q, scale4(1, cols), cols)
        assert (m.rows, m.cols, m.struct.ld, m.struct.q) == (1, cols, ld, q.data_ptr())
    assert mgn.Mat4(wide[:0, ::2], scale4(0, 64), 64).rows == 0


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("rows", [1, 2])
def test_mat8_columns_apart(rows, dtype):
    for q in spread(rows, dtype):
        if q.shape[0] == rows:
            for block in (1, 128):
                with pytest.raises(mgn.MgnError, match="adjacent"):
                    mgn.Mat8(on(q), torch.ones(1, rows if block == 1 else 1), 32, block)


def test_mat8_one_row_of_any_stride():
    wide = on(torch.zeros(5, 75, dtype=torch.float8_e4m3fn))
    for q, cols, ld in ((wide[2:3, 16:48], 20, 32), (wide[:1], 64, 80), (wide[:1, :16], 16, 16)):
        m = mgn.Mat8(q, torch.ones(1, 1), cols)
        assert (m.rows, m.cols, m.struct.ld, m.struct.q) == (1, cols, ld, q.data_ptr())
    assert mgn.Mat8(wide[:0, ::2], torch.ones(1, 0), 32).rows == 0
