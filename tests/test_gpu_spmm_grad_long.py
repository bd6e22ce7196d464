"""The product's gradients where the columns take more than one launch (tolerance: 1e-5 of the
terms' magnitudes)."""
import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def by_decoding(plan, v, o, X, dY):
    """(dvalues, its terms, dX, its terms) in 64 bits, dense matrices [M, N] on the device: where a
    retained weight stands comes from decoding its number."""
    dense = plan.decode(v, o).double()
    at = plan.decode(torch.arange(1, plan.nnz + 1, device="cuda", dtype=torch.float32), o).long()
    rows, cols = at.nonzero(as_tuple=True)
    slot = at[rows, cols] - 1
    dv, sv = (torch.zeros(plan.nnz, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(X.shape[1]):
        t = dY[rows, b].double() * X[cols, b].double()
        dv.index_add_(0, slot, t)
        sv.index_add_(0, slot, t.abs())
    d = dY.double()
    return dv, sv, dense.t() @ d, dense.t().abs() @ d.abs()


@pytest.mark.parametrize("B", [1, 3])
def test_more_columns_than_a_launch_takes(darb, B):  # noqa: F811
    N = (1 << 26) + 777
    say(f"spmm_grad: {N} columns, batch {B}")
    g = torch.Generator(device="cuda").manual_seed(B)
    plan = darb.Plan(2, N, np.full(2, 1 / 128), 0.1, darb.ROUND_FLOOR, 128, 128).upload()
    assert plan.nnz < 1 << 24                        # numbers that fp32 holds
    v, o = plan.encode(torch.randn((2, N), device="cuda", generator=g))
    X, dY = (torch.randn((n, B), device="cuda", generator=g) for n in (N, 2))
    dv, dX = plan.spmm_grad(plan.transpose(o), v, X, dY)
    wv, sv, wX, sX = by_decoding(plan, v, o, X, dY)
    assert bool(((dv - wv).abs() <= 1e-5 * sv).all())
    assert bool(((dX - wX).abs() <= 1e-5 * sX).all())
