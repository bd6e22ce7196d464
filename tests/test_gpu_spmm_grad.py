"""The gradients of the DARB product, and the column index, against the definition in 64 bits
(the products' own tolerance: 1e-5 of the terms' magnitudes)."""
import ctypes

import numpy as np
import pytest

from tests._gpu import darb, dev, host, say, torch  # noqa: F401
from tests._parity import compare

pytestmark = pytest.mark.gpu


def make(darb, rng, M, N, bs, wdtype=np.float32):  # noqa: F811
    b = rng.choice(bs, size=M)
    plan = darb.Plan(M, N, 1.0 / b, 0.1, darb.ROUND_FLOOR, min(bs), max(bs)).upload()
    W = rng.standard_normal((M, N)).astype(wdtype)
    v, o = plan.encode(dev(W))
    log2b, start, _ = (a.astype(np.int64) for a in plan.export())
    off = host(o).astype(np.int64)
    rows, cols = np.zeros(plan.nnz, np.int64), np.zeros(plan.nnz, np.int64)
    for r in range(M):
        n = -(-N // (1 << log2b[r]))
        s = slice(start[r], start[r] + n)
        rows[s] = r
        cols[s] = (np.arange(n) << log2b[r]) + off[s]
    return plan, v, o, rows, cols


def want(rows, cols, v, X, dY, N):
    X, dY, v = X.astype(np.float64), dY.astype(np.float64), v.astype(np.float64)
    dv, sv = (dY[rows] * X[cols]).sum(1), np.abs(dY[rows] * X[cols]).sum(1)
    dX, sX = np.zeros((N, X.shape[1])), np.zeros((N, X.shape[1]))
    np.add.at(dX, cols, dY[rows] * v[:, None])
    np.add.at(sX, cols, np.abs(dY[rows] * v[:, None]))
    return dv, sv, dX, sX


def index_parts(plan, index):
    raw = host(index)
    at = -(-(plan.N + 1) * 4 // 256) * 256
    starts = raw[:(plan.N + 1) * 4].view(np.uint32).astype(np.int64)
    entries = raw[at:at + 8 * plan.nnz].view(np.uint32).reshape(-1, 2).astype(np.int64)
    return starts, entries


@pytest.mark.parametrize("M,N,bs", [(1, 1, [1]), (1, 300, [128]), (70, 1, [1, 4]), (65, 127, [1, 2, 4, 8]),
                                    (300, 129, [8, 32, 128]), (513, 1000, [4, 16, 64]), (37, 5000, [1, 128]),
                                    (2000, 257, [2, 64])])
def test_index_lists_each_column_in_storage_order(darb, M, N, bs):  # noqa: F811
    rng = np.random.default_rng(M + N)
    plan, v, o, rows, cols = make(darb, rng, M, N, bs)
    say(f"transpose {M}x{N} {bs}")
    starts, entries = index_parts(plan, plan.transpose(o))
    order = np.argsort(cols, kind="stable")              # slots ascend in storage order
    assert np.array_equal(starts, np.concatenate([[0], np.cumsum(np.bincount(cols, minlength=N))]))
    assert np.array_equal(entries[:, 1], order)
    assert np.array_equal(entries[:, 0], rows[order])


@pytest.mark.parametrize("B", [1, 2, 3, 4, 5, 8, 9, 16, 20, 31, 32, 33, 64, 65, 100, 128, 150, 192, 200, 256, 257, 300, 515])
def test_spmm_grad_batches(darb, B):  # noqa: F811
    rng = np.random.default_rng(B)
    M, N = 130, 261
    plan, v, o, rows, cols = make(darb, rng, M, N, [2, 8, 32])
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    index = plan.transpose(o)
    say(f"spmm_grad B={B}")
    dv, dX = plan.spmm_grad(index, v, dev(X), dev(dY))
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, f"dvalues B={B}")
    compare(host(dX), wX, sX, 1e-5, f"dX B={B}")
    # operands inside wider buffers, at odd addresses: the same bits
    wide = lambda a: torch.nn.functional.pad(dev(a), (3, 2))[:, 3:3 + B]        # noqa: E731
    out = torch.full((N, B + 4), 5.0, device="cuda")
    dv2, dX2 = plan.spmm_grad(index, v, wide(X), wide(dY), dX=out[:, 1:B + 1])
    assert torch.equal(dv, dv2) and torch.equal(dX, dX2)
    assert bool((out[:, 0] == 5.0).all()) and bool((out[:, B + 1:] == 5.0).all())
    # one gradient at a time
    a, none = plan.spmm_grad(index, None, dev(X), dev(dY), need_X=False)
    assert none is None and torch.equal(a, dv)
    none, b = plan.spmm_grad(index, v, None, dev(dY), need_values=False)
    assert none is None and torch.equal(b, dX)


@pytest.mark.parametrize("M,N,bs,B", [(1, 1, [1], 1), (1, 300, [128], 3), (70, 1, [1, 4], 64), (40, 129, [128], 17),
                                      (1000, 64, [1], 40), (600, 2000, [4, 8, 64], 64), (5, 3000, [16], 260)])
@pytest.mark.parametrize("types", [(np.float32, np.float32), (np.float16, np.float16), (np.float16, np.float32)])
def test_spmm_grad_shapes_and_types(darb, M, N, bs, B, types):  # noqa: F811
    rng = np.random.default_rng(M + N + B)
    plan, v, o, rows, cols = make(darb, rng, M, N, bs, types[0])
    X, dY = rng.standard_normal((N, B)).astype(types[1]), rng.standard_normal((M, B)).astype(np.float32)
    say(f"spmm_grad {M}x{N} {bs} B={B} {types}")
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), dev(dY))
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, "dvalues")
    compare(host(dX), wX, sX, 1e-5, "dX")
    empty = np.setdiff1d(np.arange(N), cols)
    assert (host(dX)[empty] == 0).all()


@pytest.mark.parametrize("M,N,bs,B", [(9000, 70, [16, 64], 97), (2100, 130, [4, 32], 1100), (12300, 40, [8], 65)])
def test_spmm_grad_by_batch_tiles(darb, M, N, bs, B):  # noqa: F811
    # a dY past the L2: tiles of 64 batch columns, whose dvalues are added up afterwards, more
    # than 16 of them in several launches; a workspace whose contents do not matter
    rng = np.random.default_rng(M)
    plan, v, o, rows, cols = make(darb, rng, M, N, bs)
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    index = plan.transpose(o)
    say(f"spmm_grad tiles {M}x{N} B={B}")
    ws = torch.full((plan.nnz * 72 + plan.M * 4096 + 768,), 255, dtype=torch.uint8, device="cuda")
    dv, dX = plan.spmm_grad(index, v, dev(X), dev(dY), workspace=ws)
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, "tiles dvalues")
    compare(host(dX), wX, sX, 1e-5, "tiles dX")
    dv2, none = plan.spmm_grad(index, None, dev(X), dev(dY), need_X=False)
    assert torch.equal(dv, dv2)
    none, dX2 = plan.spmm_grad(index, v, None, dev(dY), need_values=False)
    assert torch.equal(dX, dX2)
    with pytest.raises(ValueError):
        plan.spmm_grad(index, v, dev(X), dev(dY), workspace=ws[:100])


def test_spmm_grad_one_heavy_column(darb):  # noqa: F811
    # every row keeps the same column of each block: lists of M weights, and empty ones
    rng = np.random.default_rng(1)
    M, N, B = 3000, 128, 70
    plan = darb.Plan(M, N, np.full(M, 1 / 64), 0.1, darb.ROUND_FLOOR, 64, 64).upload()
    W = np.zeros((M, N), np.float32)
    W[:, 5], W[:, 64 + 63] = rng.standard_normal(M) + 9, rng.standard_normal(M) + 9
    v, o = plan.encode(dev(W))
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    rows, cols = np.repeat(np.arange(M), 2), np.tile([5, 127], M)
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), dev(dY))
    wv, sv, wX, sX = want(rows, cols, host(v), X, dY, N)
    compare(host(dv), wv, sv, 1e-5, "heavy dvalues")
    compare(host(dX), wX, sX, 1e-5, "heavy dX")


def test_spmm_grad_infinities_stay_in_their_columns(darb):  # noqa: F811
    rng = np.random.default_rng(2)
    M, N, B = 90, 140, 13                     # lanes that take the batch's end twice
    plan, v, o, rows, cols = make(darb, rng, M, N, [4, 16])
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    dY[3, 12], dY[7, 10] = np.inf, np.nan
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), dev(dY))
    dv, dX = host(dv), host(dX)
    hit3, hit7 = rows == 3, rows == 7
    assert np.array_equal(np.isinf(dv), hit3) and np.array_equal(np.isnan(dv), hit7)
    assert np.array_equal(~np.isfinite(dX[:, 12]), np.isin(np.arange(N), cols[hit3]))
    assert np.array_equal(np.isnan(dX[:, 10]), np.isin(np.arange(N), cols[hit7]))
    assert np.isfinite(np.delete(dX, [10, 12], 1)).all()


def test_spmm_grad_by_differences(darb):  # noqa: F811
    # the product is linear: a difference over any step is its slope, up to the products' own
    # tolerance
    rng = np.random.default_rng(3)
    M, N, B = 60, 90, 12
    plan, v, o, rows, cols = make(darb, rng, M, N, [2, 8])
    X, dY = rng.standard_normal((N, B)).astype(np.float32), rng.standard_normal((M, B)).astype(np.float32)
    dv, dX = plan.spmm_grad(plan.transpose(o), v, dev(X), dev(dY))
    u, w = rng.standard_normal(plan.nnz).astype(np.float32), rng.standard_normal((N, B)).astype(np.float32)
    loss = lambda vv, XX: (host(plan.spmm(vv, o, XX)).astype(np.float64) * dY).sum()     # noqa: E731
    slope = (loss(v + dev(u), dev(X)) - loss(v - dev(u), dev(X))) / 2
    terms = np.abs(u.astype(np.float64) * (np.abs(dY)[rows] * np.abs(X)[cols]).sum(1)).sum()
    assert abs(slope - (host(dv).astype(np.float64) * u).sum()) < 4e-5 * terms
    slope = (loss(v, dev(X + w)) - loss(v, dev(X - w))) / 2
    assert abs(slope - (host(dX).astype(np.float64) * w).sum()) < 4e-5 * (np.abs(host(dX)) * np.abs(w)).sum() + \
        4e-5 * np.abs(host(v)).sum() * 10


def test_spmm_grad_stream_and_repeat(darb):  # noqa: F811
    rng = np.random.default_rng(4)
    plan, v, o, rows, cols = make(darb, rng, 700, 900, [4, 32])
    X, dY = dev(rng.standard_normal((900, 70)).astype(np.float32)), dev(rng.standard_normal((700, 70)).astype(np.float32))
    index = plan.transpose(o)
    first = plan.spmm_grad(index, v, X, dY)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    buf = torch.full_like(index, 255)
    torch.cuda.synchronize()
    again = plan.spmm_grad(plan.transpose(o, index=buf, stream=st), v, X, dY, stream=st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("bad,err", [
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"], f["dY"].half()), TypeError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"], f["dY"][:-1]), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"][:-1], f["dY"]), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"].t(), f["dY"]), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"].half(), f["dY"]), "DarbError"),
    (lambda f: f["p"].spmm_grad(f["i"][:-300], f["v"], f["X"], f["dY"]), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"][:-1], f["X"], f["dY"]), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"], f["dY"].cpu()), ValueError),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"], f["dY"], need_values=False, need_X=False), "DarbError"),
    (lambda f: f["p"].spmm_grad(f["i"], f["v"], f["X"], f["dY"], dvalues=f["v"].half()), TypeError),
    (lambda f: f["p"].transpose(f["v"]), TypeError),
    (lambda f: f["p"].transpose(f["o"][:-1]), ValueError)])
def test_spmm_grad_refusals(darb, bad, err):  # noqa: F811
    rng = np.random.default_rng(0)
    plan, v, o, rows, cols = make(darb, rng, 20, 33, [4])
    f = dict(p=plan, v=v, o=o, i=plan.transpose(o), X=torch.zeros(33, 6, device="cuda"),
             dY=torch.zeros(20, 6, device="cuda"))
    with pytest.raises(darb.DarbError if err == "DarbError" else err):
        bad(f)
