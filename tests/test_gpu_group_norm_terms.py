"""The group norm's reverse with tolerances that every term of it stands out of.

dy has a mean and a part along xhat, so that both means that the reverse subtracts, dgamma
and dbeta are as large as what is summed.  Tolerances count the additions on an element's
way into a sum instead of the elements (u = 2^-24): a thread adds up at most 128 rows (24 to
128 where a block has a sample's rows, else a 768th of all rows over the block's row
lanes: at most 11 in the cases here), neighbouring columns 3 times, a lane at most 33 of
those in LDS, 6 lanes' steps, 16 strips of a wide group; tiles are joined in 64 bits.  So
a group's sum is off by D = 192 u of the magnitudes' sum, a column's, which the row
lanes (256 at most), a tile's samples and up to 2048 blocks' parts (70 additions) make, by
Dc = 460 + samples.  The other terms are those of single roundings: xhat is off by ex = u (|mean|
rstd + 4 |xhat|) + ev |xhat|, where the mean's rounding is the same for a whole group and ev =
2 D 2^-53 (1 + (mean rstd)^2) is what 1 / std loses by the variance being a difference of 64-bit
sums (3 D 2^-53 of the squares' mean, halved, with the tiles' 64 additions); z by ez =
|gamma| ex + 3 u (|gamma xhat| + |z|), a sigmoid by (|z| + 8) u of itself.

Each case first asserts that the oracle without a term (a mean, one strip of a wide group, a
768th of the rows) lies outside the tolerance: on the CPU also without the kernels.
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2304_00338_amd import mgn  # noqa: E402

U = 2.0 ** -24
T = {"fp32": torch.float32, "bf16": torch.bfloat16}
STRIP = {"fp32": 1024, "bf16": 2048}  # columns of a wide group that a block sums at a time
EPS = 1e-5
D = 192
GPU = pytest.mark.gpu


def inputs(rows, cols, groups, dtype, spans, seed, shift, device):
    """x, gamma, beta, dy with a mean and a part along xhat."""
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=device)
    x = (normal(rows, cols) * torch.exp(0.3 * normal(1, cols)) + shift).to(T[dtype])
    gamma, beta = 1 + 0.3 * normal(cols), 0.3 * normal(cols)
    dy = 0.7 + 0.5 * normal(rows, cols)
    for a, b in spans:
        if a < b:
            dy[a:b] += 0.5 * hat(x[a:b].double(), groups)[0].float()
    return x, gamma, beta, dy.to(T[dtype])


def hat(x, groups):
    """xhat, mean and 1 / sqrt(var + eps) of one sample's rows, of each column."""
    v = x.view(x.shape[0], groups, -1)
    mean = v.mean((0, 2), keepdim=True)
    c = v - mean
    rstd = 1 / torch.sqrt((c * c).mean((0, 2), keepdim=True) + EPS)
    spread = torch.ones_like(v[:1])
    return (c * rstd).flatten(1), (mean * spread).flatten(1), (rstd * spread).flatten(1)


def oracle(x, gamma, beta, dy, groups, act, spans, less=None):
    """{name: (result, tolerance)} in 64 bits, rows outside of the samples NaN.  less: a term
    that is left out."""
    rows, cols = x.shape
    d = cols // groups
    x, gamma, beta, dy = (v.double() for v in (x, gamma, beta, dy))
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    ty, tdx = torch.zeros_like(x), torch.zeros_like(x)
    sums = torch.zeros(2, cols, dtype=torch.float64, device=x.device)
    tsums = torch.zeros_like(sums)
    for a, b in spans:
        if a >= b:
            continue
        xhat, mean, rstd = hat(x[a:b], groups)
        ex = U * (mean.abs() * rstd + 4 * xhat.abs()) + 2 * D * 2.0 ** -53 * (1 + (mean * rstd) ** 2) * xhat.abs()
        z = gamma * xhat + beta
        ez = gamma.abs() * ex + 3 * U * ((gamma * xhat).abs() + z.abs())
        t = dy[a:b]
        if act == "silu":
            sig = torch.sigmoid(z)
            y[a:b], ty[a:b] = z * sig, 1.1 * ez + (z.abs() + 10) * U * (z * sig).abs() + 2.0 ** -100
            g, eg = t * sig * (1 + z * (1 - sig)), t.abs() * (0.6 * ez + 16 * U * (1 + z.abs()) ** 2)
        else:
            y[a:b], ty[a:b] = z, ez
            g, eg = t, torch.zeros_like(t)
        keep = torch.ones_like(g)  # what the sums are of
        if less == "tile":
            keep[-max((b - a) // 768, 1):] = 0
        pairs = ((g * xhat, eg * xhat.abs() + g.abs() * ex), (g, eg))
        for i, (v, e) in enumerate(pairs):
            sums[i] += (v * keep).sum(0)
            tsums[i] += e.sum(0) + (460 + len(spans)) * U * v.abs().sum(0)
        if less is not None and less[:5] == "strip":
            for at in range(0, cols, d):
                keep[:, at + d - int(less[5:]):at + d] = 0
        means = []
        for v, e in pairs:
            def mean_of(w):
                m = w.view(b - a, groups, d).mean((0, 2), keepdim=True)
                return (m * torch.ones(1, 1, d, dtype=m.dtype, device=m.device)).flatten(1)
            w = gamma * v
            means.append((mean_of(w * keep), mean_of(gamma.abs() * e + 2 * U * w.abs()) + D * U * mean_of(w.abs())))
        (m2, em2), (m1, em1) = means
        m1, m2 = (0 * m1 if less == "m1" else m1), (0 * m2 if less == "m2" else m2)
        u, eu = gamma * g, gamma.abs() * eg + 2 * U * (gamma * g).abs()
        dx[a:b] = rstd * (u - m1 - xhat * m2)
        tdx[a:b] = rstd * (eu + em1 + xhat.abs() * em2 + ex * m2.abs() + 6 * U * (u.abs() + m1.abs() + (xhat * m2).abs())) + \
            (U + 2 * D * 2.0 ** -53 * (1 + (mean * rstd) ** 2)) * dx[a:b].abs()
    if less in ("dgamma", "dbeta"):
        sums[int(less == "dbeta")] = 0
    return {"y": (y, ty), "dx": (dx, tdx), "dgamma": (sums[0], tsums[0]), "dbeta": (sums[1], tsums[1])}


def off(got, ref, tol, bf16=False):
    """The largest share of the tolerance that a result is off by (where there is one)."""
    if bf16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    at = ~torch.isnan(ref)
    if not at.any():
        return 0.0
    r = (got.double() - ref).abs()[at] / tol[at].clamp_min(1e-300)
    return float("inf") if torch.isnan(r).any() else float(r.max())


def spans_of(rows, samples, ptr):
    n = rows // samples
    return list(zip(ptr[:-1], ptr[1:])) if ptr is not None else [(i * n, (i + 1) * n) for i in range(samples)]


def stands_out(args, ref, bf16, terms):
    """The reference without each of the terms is outside of the tolerance."""
    for less in terms:
        bad = oracle(*args, less=less)
        for name in {"dgamma": ["dgamma"], "dbeta": ["dbeta"], "tile": ["dx", "dgamma", "dbeta"]}.get(less, ["dx"]):
            share = off(bad[name][0], *ref[name], bf16 and name == "dx")
            assert share > 2, (less, name, share)


def case(rows, cols, groups, dtype, act="silu", samples=1, ptr=None, seed=0, shift=0.5, device="cuda", terms=None):
    spans = spans_of(rows, samples, ptr)
    x, gamma, beta, dy = inputs(rows, cols, groups, dtype, spans, seed, shift, device)
    args = (x, gamma, beta, dy, groups, act, spans)
    ref = oracle(*args)
    if terms is None:
        # without a strip, the last one's columns; a tile's rows where there are some
        d, s = cols // groups, STRIP[dtype]
        terms = ["m1", "m2", "dgamma", "dbeta"] + (["strip%d" % (d % s or s)] if d > s else []) + (["tile"] if rows >= 768 * len(spans) else [])
    stands_out(args, ref, dtype == "bf16", terms)
    if device != "cuda":
        return
    with_ = dict(gamma=gamma, beta=beta, act=act, eps=EPS)
    with_.update(samples=samples) if ptr is None else with_.update(sample_ptr=torch.tensor(ptr, dtype=torch.int32, device="cuda"))
    y, stats = mgn.mgn_group_norm_forward(x, groups, save=True, y=torch.full_like(x, float("nan")), **with_)
    r = mgn.mgn_group_norm_backward(x, stats, dy, groups, dx=torch.full_like(x, float("nan")), **with_)
    outside = torch.isnan(ref["y"][0])
    assert torch.isnan(y[outside]).all() and torch.isnan(r.dx[outside]).all()
    for name, got in (("y", y), ("dx", r.dx), ("dgamma", r.dgamma), ("dbeta", r.dbeta)):
        share = off(got, *ref[name], dtype == "bf16" and name in ("y", "dx"))
        print(name, round(share, 3), end=" ")
        assert share <= 1, (name, share, rows, cols, groups, dtype, act, samples, ptr and len(ptr))


# by tiles: groups narrower than a strip, of several strips with a short last one, one column each
TILES = [(2000, 2051, 7), (700, 16384, 4), (1200, 4100, 1), (900, 16384, 1), (2500, 3001, 1), (300000, 5, 1), (30001, 128, 32),
         (1500, 2048, 2048), (40000, 24, 24)]
# a block for a sample: strips of a wide group, blocks of some groups
SMALL = [(17, 2050, 1), (9, 4099, 1), (3, 16384, 1), (5, 16384, 2), (64, 128, 32), (33, 150, 10), (100, 128, 128), (600, 24, 3)]
# rows, columns, groups, samples of equal length
EVEN = [(2000, 4096, 32, 20), (424, 640, 128, 8), (6000, 2100, 1, 3), (5120, 250, 25, 10), (4200, 48, 6, 2100)]
RAGGED = [(3000, 4100, 1, [0, 0, 7, 1500, 1501, 2990]), (9000, 96, 3, [11, 4000, 4000, 8990]), (40, 4100, 2, [0, 13, 40]),
          (2000, 16384, 1, [3, 640, 2000])]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups", [(2000, 2051, 7), (200, 16384, 1), (1200, 4100, 1), (30000, 5, 1), (64, 128, 32), (17, 2050, 1)])
def test_terms_stand_out(rows, cols, groups, dtype):
    """The tolerances alone, on the CPU."""
    case(rows, cols, groups, dtype, device="cpu")


@GPU
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups", TILES + SMALL)
def test_one_sample(rows, cols, groups, dtype, act):
    case(rows, cols, groups, dtype, act, seed=rows)


@GPU
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups,samples", EVEN)
def test_equal_samples(rows, cols, groups, samples, dtype):
    case(rows, cols, groups, dtype, samples=samples, seed=rows)


@GPU
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups,ptr", RAGGED)
def test_ragged_samples(rows, cols, groups, ptr, dtype):
    case(rows, cols, groups, dtype, ptr=ptr, seed=rows)


@GPU
@pytest.mark.parametrize("shift", [1e2, 1e4, 1e6])
@pytest.mark.parametrize("rows", [60, 30000])
def test_far_mean(rows, shift):
    """A mean of many deviations shifts xhat by its rounding to float32, and costs no more; up
    to 10^4 deviations the reverse's terms are still far larger than that."""
    terms = ["m1", "m2", "dgamma", "dbeta"] if shift <= 1e4 else []
    for act in ("none", "silu"):
        case(rows, 32, 4, "fp32", act, seed=2, shift=shift, terms=terms)
    if shift == 1e2:
        case(rows, 32, 4, "bf16", seed=2, shift=shift, terms=["m1"])
