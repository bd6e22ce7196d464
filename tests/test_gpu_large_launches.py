"""The format's calls where their work takes 2^32 threads or more, which one launch does not run."""
import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_rows(darb):  # noqa: F811
    """Encode, decode, INT8 codes and packed offsets of 2^26 rows and some, two columns each."""
    M = (1 << 26) + 5
    say(f"large launches: {M} rows")
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randn((M, 2), device="cuda", generator=g)
    plan = darb.Plan(M, 2, np.full(M, 0.5), 0.5, darb.ROUND_FLOOR, 2, 2).upload()
    v, o = plan.encode(W)
    second = W[:, 1].abs() > W[:, 0].abs()           # the first of equal ones
    assert torch.equal(o, second.to(torch.uint8))
    assert torch.equal(v, torch.where(second, W[:, 1], W[:, 0]))
    W[torch.arange(M, device="cuda"), 1 - o.long()] = 0.0
    assert torch.equal(plan.decode(v, o, out=torch.full_like(W, 7.0)), W)
    codes, scales = plan.quantize_i8(v, codes=torch.zeros(M, dtype=torch.int8, device="cuda"),
                                     scales=torch.full((M,), 7.0, device="cuda"))
    assert torch.equal(codes, torch.where(v > 0, 127, -127).to(torch.int8))
    assert bool(((scales * 127 - v.abs()).abs() <= v.abs() * 2.0 ** -22).all())
    assert torch.equal(plan.unpack_offsets(plan.pack_offsets(o)), o)


def test_weights(darb):  # noqa: F811
    """Packed offsets of 2^32 weights and some."""
    M, N = (1 << 18) + 1, 1 << 15
    say(f"large launches: {M} x {N}, one weight of two")
    plan = darb.Plan(M, N, np.full(M, 0.5), 0.5, darb.ROUND_FLOOR, 2, 2).upload()
    g = torch.Generator(device="cuda").manual_seed(2)
    o = torch.randint(0, 2, (plan.nnz,), dtype=torch.uint8, device="cuda", generator=g)
    assert o.numel() > 1 << 32
    got = plan.unpack_offsets(plan.pack_offsets(o), offsets=torch.full_like(o, 9))
    assert torch.equal(got, o)


@pytest.mark.parametrize("M,B", [(16400, (1 << 17) + 1), (16, (1 << 25) + 1)])
def test_products(darb, M, B):  # noqa: F811
    """A product whose workgroups are 2^23 and more of 512 threads (X below and past 4 GiB); the
    products' tolerance: 1e-5 of the terms' magnitudes."""
    N = 65
    say(f"large launches: product {M} x {N}, batch {B}")
    g = torch.Generator(device="cuda").manual_seed(3)
    plan = darb.Plan(M, N, np.full(M, 1.0), 1.0, darb.ROUND_FLOOR, 1, 1).upload()
    v, o = plan.encode(torch.randn((M, N), device="cuda", generator=g))
    X = torch.randn((N, B), device="cuda", generator=g)
    Y = torch.full((M, B), float("nan"), device="cuda")
    assert plan.spmm(v, o, X, Y=Y) is Y
    W = plan.decode(v, o).double()
    step = (1 << 27) // M
    for b in range(0, B, step):
        x = X[:, b:b + step].double()
        assert bool(((Y[:, b:b + step] - W @ x).abs() <= 1e-5 * (W.abs() @ x.abs())).all()), b
