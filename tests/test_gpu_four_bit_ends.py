"""4-bit values at the upper end of float32: what is quantised there and read back, and
every number under the largest scales.  Values are defined to the bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402

T = {"fp32": torch.float32, "bf16": torch.bfloat16}
NUMBERS = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


@pytest.mark.parametrize("back", ["fp32", "bf16"])
@pytest.mark.parametrize("copies", ["rows", "columns"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_largest_values_read_back(dtype, copies, back):
    """Magnitudes from 3.5 x 2^126 on become 4 x 2^126, which no float is; smaller ones of the same
    32 stay finite."""
    edge = 3.5 * 2.0 ** 126
    top = float(torch.finfo(T[dtype]).max)
    below = float(np.nextafter(np.float32(edge), np.float32(0))) if dtype == "fp32" else edge * (1 - 2.0 ** -8)
    x = torch.zeros(32, 64, dtype=torch.float64)
    x[:, 0], x[:, 33] = top, -edge
    x[:, 1], x[:, 2], x[:, 3] = below, 2.0 ** 126, 0.2 * 2.0 ** 126
    x[:, 34], x[:, 35] = -below, 1.25 * 2.0 ** 126  # a middle: to the even code, 1
    x = x.to(T[dtype]).cuda()
    assert torch.isfinite(x).all() and float(x[0, 33]) == -edge
    if copies == "rows":
        m = mgn.mgn_quant4(x).rows
        got = mgn.mgn_dequant4(m, T[back])
    else:
        m = mgn.mgn_quant4(x.t().contiguous(), False, True).columns
        got = mgn.mgn_dequant4(m, T[back])
    assert (m.scale.view(torch.uint8)[0, :, :2] == 253).all()
    want = torch.zeros(32, 64, dtype=torch.float64)
    want[:, 0], want[:, 33] = float("inf"), float("-inf")
    want[:, 1], want[:, 2], want[:, 34], want[:, 35] = 3 * 2.0 ** 126, 2.0 ** 126, -3 * 2.0 ** 126, 2.0 ** 126
    assert torch.equal(got.double().cpu(), want)
    # a block whose largest is below the edge is finite
    x = torch.full((3, 32), below, dtype=torch.float64).to(T[dtype]).cuda()
    m = mgn.mgn_quant4(x).rows
    assert (m.scale.view(torch.uint8)[0, :, 0] == 252).all() and (mgn.mgn_dequant4(m, T[back]) == 6 * 2.0 ** 125).all()


@pytest.mark.parametrize("back", ["fp32", "bf16"])
def test_numbers_under_the_largest_scales(back):
    """Infinite from 2^128 on: numbers from 2 on under 2^127, 4 and 6 under 2^126, no others."""
    q = torch.arange(256, dtype=torch.uint8, device="cuda").view(16, 16).repeat(4, 1)
    s = torch.zeros(1, 64, 4, dtype=torch.uint8, device="cuda")
    s[0, :, 0] = torch.tensor([251, 252, 253, 254], device="cuda").repeat_interleave(16).to(torch.uint8)
    m = mgn.Mat4(q, s, 32)
    got = mgn.mgn_dequant4(m, T[back]).double().cpu().numpy()
    code = np.stack([q.cpu().numpy() & 15, q.cpu().numpy() >> 4], 2).reshape(64, 32)
    x = 2.0 ** (np.repeat([251, 252, 253, 254], 16) - 127.0)[:, None]
    value = NUMBERS[code & 7] * np.where(code & 8, -1, 1) * x
    number = NUMBERS[code & 7]
    infinite = ((number >= 2) & (x == 2.0 ** 127)) | ((number >= 4) & (x == 2.0 ** 126))
    assert np.array_equal(np.isinf(got), infinite)
    assert np.array_equal(got[~infinite], value[~infinite]) and np.array_equal(np.sign(got), np.sign(value))
