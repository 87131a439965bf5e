"""A training step put together from its calls: the processor's gradients of mgn_backward, one
flat buffer, clipped in place by their norm before mgn_adam_step.

The norm is summed in 64 bits and rounded once to float32 (u = 2^-24), a clipped value
once; the update is compared with the oracle's of the clipped gradients."""
import numpy as np
import pytest

import oracle as O
from gpu_util import Problem, rel_l2, segments

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2304_00338_amd import mgn  # noqa: E402

U = 2.0 ** -24


@pytest.mark.parametrize("by", ["flat", "segments", "given"])
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
def test_backward_clip_adam(prec, by):
    m = 2
    pb = Problem((7, 6, 5), m, seed=21).device()
    ctx = mgn.Context(m, pb.g.n_nodes, pb.g.n_edges, prec, save=True)
    params = pb.d_params.clone()
    grad = torch.zeros_like(params)
    n = grad.numel()
    # the list is of the buffer, whose values the steps change
    lst = mgn.TensorList([grad] if by != "segments" else [grad[a:b] for _, a, b in segments(m)])
    assert by != "segments" or sum(b - a for _, a, b in segments(m)) == n
    mm, vv = torch.zeros_like(params), torch.zeros_like(params)
    rm, rv = np.zeros(n), np.zeros(n)
    for k, part in ((1, 0.25), (2, 4.0)):  # clipped, and left as it is
        grad.zero_()
        mgn.mgn_forward(ctx, pb.dg, params, pb.d_node_in, pb.dg.efeat, save=True)
        mgn.mgn_backward(ctx, pb.d_w, grad)
        g = grad.double().cpu().numpy()
        norm = float(np.sqrt((g ** 2).sum()))
        assert np.isfinite(norm) and norm > 0
        most = part * norm
        if by == "given":
            got = mgn.mgn_grad_norm(lst)
            assert mgn.mgn_grad_clip(lst, most, norm=got) is got
        else:
            got = mgn.mgn_grad_clip(lst, most)
        assert abs(float(got) - norm) <= 1.01 * U * norm
        clipped = grad.double().cpu().numpy()
        # a given norm is a float32: one rounding more
        assert (np.abs(clipped - g * min(1.0, part)) <= (2.02 if by == "given" else 1.01) * U * np.abs(g) + 2.0 ** -149).all()
        if part > 1:
            assert np.array_equal(clipped, g)
        before = params.double().cpu().numpy()
        mgn.mgn_adam_step(mgn.Adam(), k, params, grad, mm, vv)
        rp, rm, rv = O.adam_update(before, clipped, rm, rv, k, O.lr_schedule(k - 1))
        after = params.double().cpu().numpy()
        bound = np.spacing(np.abs(rp).astype(np.float32)).astype(np.float64) + 1e-5 * np.abs(rp - before).max()
        assert (np.abs(after - rp) <= bound).all() and np.abs(after - before).max() > 0
        # the moments go on from the kernel's own
        assert rel_l2(mm.cpu().numpy(), rm) < 1e-6 and rel_l2(vv.cpu().numpy(), rv) < 1e-6
        rm, rv = mm.double().cpu().numpy(), vv.double().cpu().numpy()
