"""Rows outside of the gate groups of mgn_norm_gate_forward / _backward count
for nothing, whatever they hold: the forward itself leaves them unwritten, so
the next call finds any bits there.

Everything a call gives is compared, bit for bit, with the same call on zeros
in those rows: sizes and so the order of all sums are the same.  What that
call gives is compared with 64 bits in test_gpu_row_ops.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402

T = {"fp32": torch.float32, "bf16": torch.bfloat16}


def randn(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def both(rows, cols, xt, bt, post, pre, cuts, outside, vectors=True, gate=None):
    """(outputs with `outside` in the rows that count for nothing, outputs with
    zeros there, which rows count)."""
    at = torch.arange(rows, device="cuda")
    used = (at >= cuts[0]) & (at < cuts[-1])
    kw = dict(post=post, pre=pre, skip=0.9, scale=0.5, gate_ptr=torch.tensor(cuts, dtype=torch.int32, device="cuda"),
              gate=randn(len(cuts) - 1, cols, seed=1) if gate is None else gate)
    for i, k in enumerate(("post_gamma", "post_beta", "pre_gamma", "pre_beta")):
        if vectors and (post if i < 2 else pre) != "none":
            kw[k] = randn(cols, seed=2 + i)
    got = []
    for fill in (outside, 0.0):
        def rows_of(seed, t):
            v = randn(rows, cols, seed=seed, dtype=T[t])
            v[~used] = fill
            return v
        x, b, dy = rows_of(7, xt), rows_of(8, bt), rows_of(9, xt)
        dz = rows_of(10, bt) if pre != "none" else None
        y, z, stats = mgn.mgn_norm_gate_forward(x, b, save=True, **kw)
        stats[~used] = fill
        g = mgn.mgn_norm_gate_backward(x, b, stats, dy, dz, **kw)
        prior = mgn.NormGateGrads(None, None, *[None if t is None else torch.ones_like(t) for t in g[2:]])
        a = mgn.mgn_norm_gate_backward(x, b, stats, dy, dz, grads=prior, **kw)
        got.append(dict(y=y[used], z=None if z is None else z[used], stats=stats[used], dx=g.dx[used], db=g.db[used],
                        **{k: getattr(g, k) for k in g._fields[2:]}, **{k + " added": getattr(a, k) for k in a._fields[2:]}))
    return got[0], got[1], used


def check(*args, **kw):
    got, want, used = both(*args, **kw)
    for k, v in want.items():
        assert (got[k] is None) == (v is None), k
        if v is not None:
            assert v.isfinite().all() and torch.equal(got[k], v), (k, args)
    return got


# each way to hold a row: 16, 32 and 64 lanes, a block with one and with two runs of 8 a lane
WIDTHS = [3, 128, 150, 250, 512, 600, 1500, 5000, 5200, 8200]
CUTS = [[7, 100, 100, 271], [0, 33, 250], [40, 40, 41, 300], [299, 300], [0, 1]]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("outside", [float("nan"), float("inf"), float("-inf"), 3.0e38])
def test_any_value_outside(cols, outside):
    for cuts in CUTS:
        check(300, cols, "fp32", "bf16", "layer", "rms", cuts, outside)
    check(300, cols, "bf16", "bf16", "rms", "layer", CUTS[0], outside)


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("xt,bt", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
def test_any_norm(post, pre, xt, bt):
    for cols in (128, 600):
        for vectors in (True, False):
            check(300, cols, xt, bt, post, pre, CUTS[0], float("nan"), vectors)


@pytest.mark.parametrize("cols", [128, 200, 512, 600])
def test_walkers_of_many_rows(cols):
    """Counted rows and others in one walker, whose rows are many here; the last row, which
    walkers past the end look at, among the others."""
    check(50001, cols, "fp32", "bf16", "layer", "layer", [3, 777, 777, 20000, 49990], float("nan"))
    check(50001, cols, "bf16", "bf16", "rms", "rms", [25000, 25001], float("inf"))


def test_no_row_counts():
    for cols in (128, 600):
        for cuts in ([5, 5], [300, 300], [0, 0, 0]):
            got = check(300, cols, "fp32", "fp32", "layer", "rms", cuts, float("nan"))
            assert not any(got[k].any() for k in ("dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta"))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_gate_of_an_empty_group(value):
    """A gate that no row has reaches no gradient but its own, which is 0."""
    for cols in (128, 600):
        for cuts in ([60, 60, 200, 200], [60, 200, 200, 250]):
            gate = randn(3, cols, seed=1)
            empty = [i for i in range(3) if cuts[i] == cuts[i + 1]]
            gate[empty] = value
            got = check(300, cols, "fp32", "fp32", "layer", "rms", cuts, float("nan"), gate=gate)
            assert not got["dgate"][empty].any()
