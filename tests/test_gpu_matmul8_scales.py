"""mgn_matmul8 with scales over all of float32: a result that float32 holds is
right also where the product of its two scales is not a normal float32.

Tolerance, against 64 bits: as for ordinary scales (K + K/128 + 8) steps of
2u = 2^-23 of the terms' magnitudes (a block's sum takes two more roundings, of
the 8, where its scales are taken apart), a bfloat16 result the cuts of the 8-bit
instruction, 7 2^-13 of the magnitudes, and 2^-8 of itself; and, where numbers
are subnormal, half a step of 2^-149 for each block's product and sum and for
the result."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402

U = 2.0 ** -24
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
# sizes of every way to sum: up to 16 and 32 rows, tiles, tiles with the sums split, large tiles
SIZES = [(1, 300, 384), (16, 40, 2500), (20, 90, 384), (40, 200, 384), (130, 140, 700), (64, 64, 20000), (64, 200, 128)]
LARGE = (4096, 3840, 1100)


def numbers(r, c, fmt, small, seed):
    """8-bit numbers; small: the format's few least ones."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.zeros(r, -(-c // 16) * 16, dtype=torch.uint8, device="cuda")
    top = 4 if small else {"e4m3": 0x7e, "e5m2": 0x7b}[fmt]
    n = torch.randint(0, top + 1, (r, c), generator=g, device="cuda", dtype=torch.uint8)
    q[:, :c] = n + 128 * torch.randint(0, 2, (r, c), generator=g, device="cuda", dtype=torch.uint8)
    return q.view(F8[fmt])


def matrix(r, c, fmt, block, small, exponents, seed):
    """Scales 2^e (1 + [0, 1)), e one of exponents for each block."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    shape = (-(-c // 128), -(-r // block))
    e = torch.tensor(exponents, device="cuda", dtype=torch.float64)
    e = e[torch.randint(0, len(exponents), shape, generator=g, device="cuda")]
    s = torch.exp2(e) * (1 + torch.rand(shape, generator=g, device="cuda", dtype=torch.float64) * 0.99)
    return mgn.Mat8(numbers(r, c, fmt, small, seed), s.float().contiguous(), c, block)


def values(m):
    v = m.q[:, :m.cols].float().double()
    s = m.scale.double().t().repeat_interleave(m.block_rows, 0)[:m.rows].repeat_interleave(128, 1)[:, :m.cols]
    return v * s


def check(a, b, dtype):
    out = mgn.mgn_matmul8(a, b, dtype=dtype).double()
    A, B = values(a), values(b)
    ref, mag = A @ B.t(), A.abs() @ B.abs().t()
    tol = (a.cols + a.cols / 128 + 8) * 2 * U * mag + (2 * (-(-a.cols // 128)) + 2) * 2.0 ** -149
    if dtype == torch.bfloat16:
        tol = tol + 7 * 2.0 ** -13 * mag
        tol = tol + 2.0 ** -8 * (ref.abs() + tol) + 2.0 ** -134
    held = mag < 2.0 ** 127  # no sum on the way leaves float32 either
    bad = held & ~((out - ref).abs() <= tol)
    assert not bad.any(), (a.rows, b.rows, a.cols, int(bad.sum()), bad.nonzero()[:3].tolist(), out[bad][:3].tolist(),
                           ref[bad][:3].tolist())
    normal = held & (mag > 2.0 ** -100)
    return held.float().mean().item(), normal.float().mean().item()


ANY = [-126, -110, -95, -64, -40, -8, 0, 8, 40, 64, 95, 110, 118]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("ba,bb", [(1, 128), (1, 1), (128, 128), (128, 1)])
def test_scales_of_any_size(dtype, fa, fb, ba, bb):
    for i, (m, n, k) in enumerate(SIZES):
        for small in (False, True):
            a, b = matrix(m, k, fa, ba, small, ANY, 2 * i), matrix(n, k, fb, bb, small, ANY, 2 * i + 1)
            check(a, b, dtype)
            # both low, and both high: products of scales below 2^-126, and infinite
            low = check(matrix(m, k, fa, ba, False, [-72, -66], 2 * i), matrix(n, k, fb, bb, False, [-70, -62], 2 * i + 1), dtype)
            assert low[0] == 1
            high = check(matrix(m, k, fa, ba, True, [64, 60], 2 * i), matrix(n, k, fb, bb, True, [65, 66], 2 * i + 1), dtype)
            if fa == fb == "e5m2":
                assert high[1] > 0.9, high  # numbers up to 2^-14: 2^-28 2^131 K


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fa", ["e4m3", "e5m2"])
def test_scales_of_any_size_large_tiles(dtype, fa):
    m, n, k = LARGE
    check(matrix(m, k, fa, 1, False, [-72, -20, 0], 1), matrix(n, k, "e4m3", 128, False, [-70, -40, 3], 2), dtype)
    check(matrix(m, k, fa, 1, True, ANY, 1), matrix(n, k, "e4m3", 128, True, ANY, 2), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bb", [1, 128])
def test_zero_blocks_under_huge_scales(dtype, bb):
    """Blocks whose numbers meet only zeros give 0, not a NaN."""
    for m, n, k in SIZES + [LARGE]:
        a, b = matrix(m, k, "e4m3", 1, False, [70], 1), matrix(n, k, "e4m3", bb, False, [70], 2)
        a.q.view(torch.uint8)[:, 0::2] = 0
        b.q.view(torch.uint8)[:, 1::2] = 0
        assert (mgn.mgn_matmul8(a, b, dtype=dtype) == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bb", [1, 128])
def test_rows_apart(dtype, bb):
    """Rows of zeros, of tiny, huge and no numbers leave the other rows' bits as they are."""
    for m, n, k in SIZES + [LARGE]:
        g = torch.Generator(device="cuda").manual_seed(m)
        x, w = torch.randn(m, k, generator=g, device="cuda"), torch.randn(n, k, generator=g, device="cuda")
        b = mgn.mgn_quant8(w * 1e-3, "e4m3", bb).rows
        want = mgn.mgn_matmul8(mgn.mgn_quant8(x).rows, b, dtype=dtype)
        other = torch.zeros(m, dtype=torch.bool, device="cuda")
        for i, v in enumerate((0.0, 1e-37, 3e38, float("nan"))):
            x[2 * i + 1::11] = v
            other[2 * i + 1::11] = True
        got = mgn.mgn_matmul8(mgn.mgn_quant8(x).rows, b, dtype=dtype)
        assert torch.equal(got[~other], want[~other])
        assert (got[1::11] == 0).all() and got[7::11].isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bb", [1, 128])
def test_zero_negative_and_subnormal_scales(dtype, bb):
    """Scales that mgn_quant8 does not write, but a Mat8 may hold."""
    for m, n, k in SIZES + [LARGE]:
        a, b = matrix(m, k, "e4m3", 1, False, [-3, 0, 5], 1), matrix(n, k, "e4m3", bb, False, [-2, 1, 100], 2)
        flat = a.scale.view(-1)
        flat[0::5] = 0.0
        flat[1::5] *= -1
        flat[2::5] = 3 * 2.0 ** -149
        flat[3::5] = -(2.0 ** -130)
        b.scale.view(-1)[0::3] *= -1
        check(a, b, dtype)
