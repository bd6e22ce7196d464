"""The product's gradients where the columns take more than one launch, and where offsets pass 24
and 32 bits: rows of dY far apart, or many (tolerance: 1e-5 of the terms' magnitudes)."""
import numpy as np
import pytest

from tests._gpu import darb, dev, host, say, torch  # noqa: F401
from tests._parity import compare
from tests.test_gpu_spmm_grad import make, want

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


def test_rows_past_24_bits(darb):  # noqa: F811
    M = (1 << 24) + 5                                # offsets of 64 bits
    say(f"spmm_grad: {M} rows")
    g = torch.Generator(device="cuda").manual_seed(7)
    plan = darb.Plan(M, 3, np.full(M, 1 / 4), 0.25, darb.ROUND_FLOOR, 4, 4).upload()
    v, o = plan.encode(torch.randn((M, 3), device="cuda", generator=g))
    X, dY = (torch.randn((n, 1), device="cuda", generator=g) for n in (3, M))
    dv, dX = plan.spmm_grad(plan.transpose(o), v, X, dY)
    # one weight a row, in the rows' order
    cols = o.long()
    assert bool(((dv - dY[:, 0].double() * X[cols, 0].double()).abs() <= 1e-5 * dv.abs() + 1e-30).all())
    for c in range(3):
        t = (v.double() * dY[:, 0].double())[cols == c]
        assert abs(dX[c, 0].item() - t.sum().item()) <= 1e-5 * t.abs().sum().item()


@pytest.mark.parametrize("ld", [(1 << 22) - 1, 1 << 22])
@pytest.mark.parametrize("B", [1, 3, 4, 7, 20, 64, 100, 150, 300])
def test_rows_of_dy_far_apart(darb, B, ld):  # noqa: F811
    """The last leading dimension whose bytes take 24 bits, and the first that does not."""
    say(f"spmm_grad: batch {B}, leading dimension {ld}")
    rng = np.random.default_rng(B)
    M, N = 8, 150
    plan, v, o, rows, cols = make(darb, rng, M, N, [2, 8])
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    far = torch.full((M * ld,), float("nan"), device="cuda").view(M, ld)[:, :B]
    far.copy_(dev(dY))
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), far)
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, f"dvalues B={B}")
    compare(host(dX), wX, sX, 1e-5, f"dX B={B}")


@pytest.mark.parametrize("M", [256, 257])
@pytest.mark.parametrize("B", [1, 64, 260])
def test_rows_of_dy_to_4_gib(darb, M, B):  # noqa: F811
    """The last dY whose byte offsets take 32 bits, and the first that does not."""
    ld = (1 << 22) - 1
    assert (M * ld < 1 << 30) == (M == 256)
    say(f"spmm_grad: {M} rows of batch {B}, leading dimension {ld}")
    rng = np.random.default_rng(M + B)
    N = 90
    plan, v, o, rows, cols = make(darb, rng, M, N, [4, 16])
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    far = torch.empty(M * ld, device="cuda").view(M, ld)[:, ld - B:]             # to its very end
    far.copy_(dev(dY))
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), far)
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, f"dvalues M={M} B={B}")
    compare(host(dX), wX, sX, 1e-5, f"dX M={M} B={B}")
