"""Gate groups of mgn_norm_gate_forward / _backward where many of them are empty
and a walker's rows, several each, lie on both sides.

The time such a call takes is bounded by the steps of a search, which shows
here only in that the calls end; what they give is compared with the same
groups without the empty ones, bit for bit (the sums' order goes by the rows)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402


def randn(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def run(x, b, dy, dz, gate, ptr):
    kw = dict(post="layer", pre="rms", gate=gate, gate_ptr=ptr)
    y, z, stats = mgn.mgn_norm_gate_forward(x, b, save=True, **kw)
    return y, z, mgn.mgn_norm_gate_backward(x, b, stats, dy, dz, **kw)


# rows: four or more to a walker of 16 lanes, 20 or more to a block
@pytest.mark.parametrize("rows,cols,n", [(70001, 8, 2 ** 22 + 5), (20011, 600, 2 ** 16 + 3)])
def test_empty_groups_between_rows_of_a_walker(rows, cols, n):
    # group sizes; the empty ones between them: none, one, two and very many
    sizes = [rows // 3 + 1, 1, 2, rows // 5, rows // 7, 1, 1, 7]
    sizes.append(rows - sum(sizes))
    gaps = [0, 1, 2, 3, n // 2, 17, 0, n // 4]
    place = [sum(gaps[:i]) + i for i in range(len(sizes))]
    place = [p + 5 for p in place]  # empty ones in front too
    count = torch.zeros(n, dtype=torch.int64, device="cuda")
    count[torch.tensor(place, device="cuda")] = torch.tensor(sizes, device="cuda")
    ptr = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32)
    near = torch.tensor([0] + sizes, device="cuda").cumsum(0).to(torch.int32)
    gate = randn(n, cols, seed=1)
    x, b, dy, dz = (randn(rows, cols, seed=s) for s in (2, 3, 4, 5))
    y, z, g = run(x, b, dy, dz, gate, ptr)
    y2, z2, g2 = run(x, b, dy, dz, gate[place].contiguous(), near)
    assert torch.equal(y, y2) and torch.equal(z, z2) and torch.equal(g.dx, g2.dx) and torch.equal(g.db, g2.db)
    assert torch.equal(g.dgate[place], g2.dgate)
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[place] = False
    assert not g.dgate[rest].any()


@pytest.mark.parametrize("cols", [16, 600])
def test_every_other_group_empty(cols):
    rows = 50000
    ptr = torch.arange(rows + 1, device="cuda").repeat_interleave(2)[1:].to(torch.int32)  # 0 1 1 2 2 ... rows rows
    n = ptr.numel() - 1
    gate = randn(n, cols, seed=1)
    x, b, dy, dz = (randn(rows, cols, seed=s) for s in (2, 3, 4, 5))
    y, z, g = run(x, b, dy, dz, gate, ptr)
    own = gate[0::2].contiguous()
    assert own.shape[0] == rows
    kw = dict(post="layer", pre="rms", gate=own)  # a gate for each row
    y2, z2, st = mgn.mgn_norm_gate_forward(x, b, save=True, **kw)
    g2 = mgn.mgn_norm_gate_backward(x, b, st, dy, dz, **kw)
    assert torch.equal(y, y2) and torch.equal(z, z2) and torch.equal(g.dx, g2.dx) and torch.equal(g.db, g2.db)
    assert torch.equal(g.dgate[0::2], g2.dgate) and not g.dgate[1::2].any()
