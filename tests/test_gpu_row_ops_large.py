"""The row operators' kernels that only large calls take, on both sides of each border: the 4-bit
quantiser's tiles from 128 MB of x on and its column sums in two steps from 1025 blocks of 128
rows on, reading back and the group norm's results past L2 from 32 MB of aligned rows on,
and the 256 x 256 product with every epilogue.  Plain implementations in 64 bits on the
device.

Numbers, scales and read values are compared for equality.  A column sum is 8 rows of a
thread, 2 steps over lanes, 3 waves, then 256 / 64 + 16 and 9 / 64 + 16 additions: under 56 u of the
magnitudes' sum (u = 2^-24), which has a mean of its rows' size, so that a block that is left
out (1/1026 and more of it) stands out; one more for what is there.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402
from test_gpu_group_norm_terms import case as group_norm_case  # noqa: E402

U = 2.0 ** -24
T = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}


def randn(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def oracle4(x):
    """(codes [rows][cols up to 32], scale bytes [rows][blocks]) of float rows; no negative zeros."""
    r, c = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -c % 32)).view(r, -1, 32)
    bad = ~torch.isfinite(v).all(2)
    v = torch.where(bad[:, :, None], 0.0, v)
    frac, e = torch.frexp(v.abs().amax(2))
    e = torch.where(v.abs().amax(2) > 0, (e - 3 + (frac >= 0.875).int()).clamp_min(-127), -127)
    t = (v * torch.exp2(-e.double())[:, :, None]).flatten(1)
    mid = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    lo, hi = (torch.bucketize(t.abs(), mid, right=k) for k in (False, True))  # differ at a middle
    code = torch.where(lo % 2 == 0, lo, hi)
    code = torch.where((t < 0) & (code > 0), code + 8, code)
    return code.to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


def check_mat4(m, x, what):
    r, c = x.shape
    code, s = oracle4(x)
    q = torch.stack([m.q & 15, m.q >> 4], 2).flatten(1)
    q = torch.where(q == 8, 0, q)
    assert (m.rows, m.cols, q.shape) == (r, c, code.shape), what
    assert torch.equal(q, code), (what, (q != code).nonzero()[:4].tolist())
    got = m.scale.view(torch.uint8).transpose(0, 1).flatten(1)
    assert torch.equal(got[:, :s.shape[1]], s) and not got[:, s.shape[1]:].any(), what


LIMIT = 128 << 20
# rows, columns, whether x is larger than the border
QUANT = {"fp32": [(131203, 255, False), (131203, 259, True), (262144, 128, False), (262177, 128, True)],
         "bf16": [(131203, 511, False), (131203, 515, True), (131073, 512, True)]}


@pytest.mark.parametrize("dtype,rows,cols,large", [(t, *s) for t, v in QUANT.items() for s in v])
def test_quant4(dtype, rows, cols, large):
    assert (rows * cols * SIZE[dtype] > LIMIT) == large and rows > 1024 * 128 or not large
    x = (randn(rows, cols, seed=cols) * torch.exp(randn(rows, 1, seed=cols + 1)) + 0.5).to(T[dtype])
    x[rows - 1, cols - 1], x[70000, 40], x[300, 0] = float("inf"), float("nan"), 0.0
    out = mgn.mgn_quant4(x, True, True)
    check_mat4(out.rows, x, "rows")
    columns = out.columns
    del out
    check_mat4(columns, x.t().contiguous(), "columns")
    # with sums; an infinity and a NaN reach their columns' only
    before = randn(cols, seed=9) * 1e4
    again = mgn.mgn_quant4(x, True, True, colsum=before.clone(), accumulate=True)
    assert torch.equal(again.columns.q, columns.q) and torch.equal(again.columns.scale.view(torch.uint8), columns.scale.view(torch.uint8))
    alone = mgn.mgn_quant4(x, True, False)  # the kernel for rows only
    assert torch.equal(again.rows.q, alone.rows.q)
    assert torch.equal(again.rows.scale.view(torch.uint8), alone.rows.scale.view(torch.uint8))
    ref, mag = x.double().sum(0), x.double().abs().sum(0)
    tol = 56 * U * mag + 2 * U * (ref.abs() + before.double().abs())
    fine = torch.isfinite(ref)
    assert int((~fine).sum()) == 2 and torch.equal(torch.isfinite(again.colsum), fine)
    off = (again.colsum.double() - ref - before.double()).abs()
    assert (off[fine] <= tol[fine]).all(), float((off / tol)[fine].max())
    assert (x[:128].double().sum(0).abs()[fine] > 2 * tol[fine]).any()  # a block that is left out


@pytest.mark.parametrize("dtype,rows,cols,ld,large", [
    ("fp32", 33003, 259, 260, True), ("fp32", 33003, 259, 261, False), ("fp32", 32000, 260, 260, False),
    ("bf16", 65803, 259, 264, True), ("bf16", 65803, 259, 266, False), ("bf16", 64001, 260, 264, False), ("bf16", 132001, 128, 128, True)])
def test_dequant4(dtype, rows, cols, ld, large):
    assert (rows * cols * SIZE[dtype] > 32 << 20 and ld * SIZE[dtype] % 16 == 0) == large
    m = mgn.mgn_quant4(randn(rows, cols, seed=1) * torch.exp(3 * randn(rows, 1, seed=2))).rows
    m.scale.view(torch.uint8)[0, 1000, 1] = 255
    big = torch.full((rows + 1, ld), 7.0, dtype=T[dtype], device="cuda")
    mgn.mgn_dequant4(m, out=big[:rows, :cols])
    q = torch.stack([m.q & 15, m.q >> 4], 2).flatten(1)[:, :cols].long()
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    s = m.scale.view(torch.uint8).transpose(0, 1).flatten(1).double()
    ref = table[q & 7] * (1 - 2 * (q >> 3)) * torch.where(s == 255, float("nan"), torch.exp2(s - 127)).repeat_interleave(32, 1)[:, :cols]
    got = big[:rows, :cols].double()
    bad = torch.isnan(ref)
    assert int(bad.sum()) == 32 and torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], ref[~bad])
    assert (big[rows] == 7).all() and (big[:, cols:] == 7).all()


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype,rows,cols,groups", [("bf16", 66001, 256, 32), ("bf16", 65000, 256, 32), ("bf16", 64900, 259, 37),
                                                    ("bf16", 4200, 4104, 27), ("fp32", 33001, 256, 32), ("fp32", 32700, 256, 32)])
def test_group_norm(dtype, rows, cols, groups, act):
    """Results of more than 32 MB and of less, of aligned rows and of others; samples that end
    anywhere and rows outside of them."""
    case_ = dict(act=act, ptr=[5, 5, rows // 3, rows // 3 + 1, rows - 7], terms=["m1", "m2", "dgamma", "dbeta"])
    group_norm_case(rows, cols, groups, dtype, seed=cols, **case_)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_group_norm_strides(dtype):
    """Aligned rows inside wider ones, and unaligned ones, as the same rows alone."""
    rows, cols = 66001, 264
    x, dy, g, b = randn(rows, cols, seed=1).to(T[dtype]), randn(rows, cols, seed=2).to(T[dtype]), randn(cols, seed=3), randn(cols, seed=4)
    with_ = dict(gamma=g, beta=b, act="silu", samples=1)
    y, st = mgn.mgn_group_norm_forward(x, 33, save=True, **with_)
    r = mgn.mgn_group_norm_backward(x, st, dy, 33, **with_)
    for ld, at in ((272, 8), (267, 1)):
        wide = torch.full((rows, ld), 7.0, dtype=T[dtype], device="cuda")
        out = wide[:, at:at + cols]
        assert torch.equal(mgn.mgn_group_norm_forward(x, 33, y=out, **with_)[0], y)
        assert (wide[:, :at] == 7).all() and (wide[:, at + cols:] == 7).all()
        out.copy_(dy)
        again = mgn.mgn_group_norm_backward(x, st, out, 33, dx=out, **with_)  # in dy's place
        assert all(torch.equal(p, q) for p, q in zip(again, r))
        assert (wide[:, :at] == 7).all() and (wide[:, at + cols:] == 7).all()


@pytest.mark.parametrize("by", ["samples", "sample_ptr"])
@pytest.mark.parametrize("n,groups,d", [(1 << 21, 2, 4), (1 << 17, 1024, 1)])
def test_group_norm_most_samples(n, groups, d, by):
    """The largest number of samples, and of samples times 32 groups.  Sums of 8 or 2 values, and
    six roundings more, under 64 u of the magnitudes; xhat is off by u (|mean| rstd + 4 |xhat|).  A
    column's sum is of 1024 samples a block (one of 2048) or 2731 (a 768th), 256 row lanes and 50
    additions more."""
    rows, cols, eps = 2 * n, groups * d, 1e-2
    blocks, depth = (2048, 1330) if by == "samples" else (768, 3040)
    x, dy = randn(rows, cols, seed=1), 0.7 + randn(rows, cols, seed=2)
    g, b = 1 + 0.3 * randn(cols, seed=3), randn(cols, seed=4)

    def split(v):
        return v.double().view(n, 2, groups, d)

    def mean_of(v):
        return v.mean((1, 3), keepdim=True)
    mean = mean_of(split(x))
    rstd = 1 / torch.sqrt(mean_of((split(x) - mean) ** 2) + eps)
    xhat = (split(x) - mean) * rstd
    ex = U * (mean.abs() * rstd + 4 * xhat.abs())
    gv, bv = g.double().view(1, 1, groups, d), b.double().view(1, 1, groups, d)
    u = split(dy) * gv
    m2 = mean_of(u * xhat)
    dx = rstd * (u - mean_of(u) - xhat * m2)
    tdx = rstd * (64 * U * (u.abs() + mean_of(u.abs()) + xhat.abs() * mean_of((u * xhat).abs())) + ex * m2.abs() +
                  xhat.abs() * mean_of(u.abs() * ex))
    with_ = dict(gamma=g, beta=b, eps=eps)
    with_.update(samples=n) if by == "samples" else with_.update(sample_ptr=torch.arange(0, rows + 1, 2, dtype=torch.int32, device="cuda"))
    y, st = mgn.mgn_group_norm_forward(x, groups, save=True, **with_)
    r = mgn.mgn_group_norm_backward(x, st, dy, groups, **with_)
    assert ((split(y) - xhat * gv - bv).abs() <= gv.abs() * ex + 4 * U * ((gv * xhat).abs() + bv.abs())).all()
    assert ((split(r.dx) - dx).abs() <= tdx).all()
    for got, v, e in ((r.dgamma, split(dy) * xhat, split(dy).abs() * ex), (r.dbeta, split(dy), 0 * ex)):
        ref, tol = v.view(rows, cols).sum(0), depth * U * v.abs().view(rows, cols).sum(0) + e.view(rows, cols).sum(0)
        assert ((got.double() - ref).abs() <= tol).all()
    # a block's samples would be missed
    assert (split(dy)[:n // blocks].sum((0, 1)).abs() > 2 * depth * U * split(dy).abs().sum((0, 1))).any()


# ------------------------------------------- 256 x 256 products with an epilogue
def values(m):
    q = torch.stack([m.q & 15, m.q >> 4], 2).flatten(1)[:, :m.cols].long()
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    s = m.scale.view(torch.uint8).transpose(0, 1).flatten(1).double()
    return table[q & 7] * (1 - 2 * (q >> 3)) * torch.exp2(s - 127).repeat_interleave(32, 1)[:, :m.cols]


@pytest.mark.parametrize("act", ["none", "relu", "relu_grad"])
@pytest.mark.parametrize("m,n,k", [(4096, 3841, 1100), (3841, 4096, 1024), (4090, 4095, 300)])
def test_matmul4_large_tiles_epilogue(m, n, k, act):
    """k / 32 block sums of one step 2u each of the magnitudes' sum, as many as 24 more, one
    for a bias and one for what is there; bf16 2^-8 of itself."""
    a, b = (mgn.mgn_quant4(randn(r, k, seed=s) * torch.exp(randn(r, 1, seed=s + 1))).rows for r, s in ((m, 1), (n, 3)))
    va, vb = values(a), values(b)
    plain, mag = va @ vb.t(), va.abs() @ vb.abs().t()
    bias = randn(n, seed=5) * 30
    for dtype in ("fp32", "bf16"):
        for bias_, at, add, ld in ((bias, "fp32", False, n), (None, "bf16", True, n + 7), (bias, "bf16", True, -(-n // 8) * 8)):
            aux = randn(m, n + 3, seed=6).to(T[at])[:, 2:n + 2] if act == "relu_grad" else None
            wide = torch.full((m + 1, ld), float("nan"), dtype=T[dtype], device="cuda")
            out = wide[:m, :n]
            ref, tol = plain.clone(), (k / 32 + 24) * 2 * U * mag
            if bias_ is not None:
                ref, tol = ref + bias_.double(), tol + 2 * U * (mag + bias_.double().abs())
            if act == "relu":
                ref.clamp_(min=0)
            elif act == "relu_grad":
                on = (aux > 0).double()
                ref, tol = ref * on, tol * on
            if add:
                out.copy_(randn(m, n, seed=7) * 10)
                ref, tol = ref + out.double(), tol + 2 * U * (ref.abs() + out.double().abs())
            mgn.mgn_matmul4(a, b, bias=bias_, act=act, aux=aux, out=out, accumulate=add)
            if dtype == "bf16":
                tol = tol + 2.0 ** -8 * (ref.abs() + tol)
            off = (out.double() - ref).abs() - tol
            assert (off <= 0).all(), (dtype, at, add, ld, float(off.max()), (off > 0).nonzero()[:4].tolist())
            assert torch.isnan(wide[m].float()).all() and torch.isnan(wide[:, n:].float()).all()
