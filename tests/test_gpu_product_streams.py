"""The format's calls on a given stream, beside work that waits on the current one: no call's memory
is another's (different inputs on the two streams, buffers of one size)."""
import numpy as np
import pytest

from tests._gpu import darb, dev, say, torch  # noqa: F401
from tests._streams import Busy, copies, flat, same, without_native

pytestmark = pytest.mark.gpu

H, T, BATCH, I = 32, 5, 4, 24


def inputs(d, seed):
    rng = np.random.default_rng(seed)
    M, N, B = 300, 260, 70
    b = np.random.default_rng(0).choice([4, 16], size=M)          # one pattern of sizes
    plan = d.Plan(M, N, 1.0 / b, 0.1, 0, 4, 16).upload()
    W = dev(rng.standard_normal((M, N)).astype(np.float32))
    v, o = plan.encode(W)
    q, s = plan.quantize_i8(v)
    f = dict(plan=plan, W=W, v=v, o=o, p=plan.pack_offsets(o), q=q, s=s,
             x=dev(rng.standard_normal(N).astype(np.float32)), X=dev(rng.standard_normal((N, B)).astype(np.float32)))
    for name, n in (("wih", I), ("whh", H)):
        p = d.Plan(4 * H, n, np.full(4 * H, 0.25), 0.25, 0, 4, 4).upload()
        f[name] = (p, *p.encode(dev(rng.standard_normal((4 * H, n)).astype(np.float32))))
    f["seq"] = dev(rng.standard_normal((I, T * BATCH)).astype(np.float32))
    f["counts"] = dev(rng.integers(1, N // 4, M))
    return f


def planned(d, f, **k):
    p = d.Plan.from_device_counts(f["plan"].N, f["counts"], int(f["counts"].sum()), 0, 4, 64, **k)
    return [torch.from_numpy(np.array(t)).cuda() for t in p.export()] + [p.encode(f["W"])[0]]


CALLS = {
    "encode": lambda d, f, **k: f["plan"].encode(f["W"], **k),
    "decode": lambda d, f, **k: f["plan"].decode(f["v"], f["o"], **k),
    "spmv": lambda d, f, **k: f["plan"].spmv(f["v"], f["o"], f["x"], **k),
    "spmm": lambda d, f, **k: f["plan"].spmm(f["v"], f["o"], f["X"], **k),
    "pack": lambda d, f, **k: f["plan"].pack_offsets(f["o"], **k),
    "unpack": lambda d, f, **k: f["plan"].unpack_offsets(f["p"], **k),
    "spmv_packed": lambda d, f, **k: f["plan"].spmv_packed(f["v"], f["p"], f["x"], **k),
    "spmm_packed": lambda d, f, **k: f["plan"].spmm_packed(f["v"], f["p"], f["X"], **k),
    "quantize": lambda d, f, **k: f["plan"].quantize_i8(f["v"], **k),
    "spmv_i8": lambda d, f, **k: f["plan"].spmv_i8(f["q"], f["s"], f["x"], offsets=f["o"], **k),
    "spmm_i8": lambda d, f, **k: f["plan"].spmm_i8(f["q"], f["s"], f["X"], packed=f["p"], **k),
    "prune": lambda d, f, **k: d.prune_counts(f["W"], 5000, **k),
    "lstm": lambda d, f, **k: d.lstm_layer(f["wih"], f["whh"], f["seq"], H, T, BATCH, **k),
}


@pytest.fixture(scope="module")
def busy(darb):  # noqa: F811
    return Busy()


@pytest.fixture(scope="module")
def pair(darb):  # noqa: F811
    return inputs(darb, 1), inputs(darb, 2)


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_memory_of_two_streams(darb, busy, pair, monkeypatch, name, path):  # noqa: F811
    say(f"memory of two streams: {name} {path}")
    if path == "python":                             # nothing that the native module takes
        without_native(monkeypatch, darb)
    call, (fa, fb) = CALLS[name], pair
    want_a, want_b = copies(call(darb, fa)), copies(call(darb, fb))
    assert not same(want_a, want_b)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    # the current stream's results and workspace are free for its next calls, not for st's
    busy.queue()
    got_a = copies(call(darb, fa))
    r = call(darb, fb, stream=st)
    # st's results are used here, then free: st's next call waits with their memory
    torch.cuda.current_stream().wait_stream(st)
    busy.queue()
    got_b = copies(r)
    del r
    again = call(darb, fa, stream=st)
    torch.cuda.synchronize()
    assert same(got_a, want_a) and same(got_b, want_b) and same(flat(again), want_a)


def test_plans_made_for_a_given_stream(darb, busy, pair):  # noqa: F811
    """A plan's tables lie in the current stream's memory, which the given stream waits for."""
    say("plans made for a given stream")
    fa, fb = pair
    want_a, want_b = planned(darb, fa), planned(darb, fb)
    up = darb.Plan(300, 260, np.full(300, 0.1), 0.1, 0, 4, 16).upload()
    want_v = up.encode(fa["W"])[0]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy.queue()
    junk = [torch.full((n,), 85, dtype=torch.uint8, device="cuda")
            for n in (fa["plan"].workspace.numel(), up.workspace.numel())]
    del junk
    got_b = planned(darb, fb, stream=st)
    busy.queue()
    junk = torch.full_like(up.workspace, 85)
    del junk
    again = darb.Plan(300, 260, np.full(300, 0.1), 0.1, 0, 4, 16).upload(stream=st)
    got_v = again.encode(fa["W"])[0]
    torch.cuda.synchronize()
    assert same(got_b, want_b) and torch.equal(got_v, want_v) and same(planned(darb, fa), want_a)


def test_the_current_stream_named(darb, pair):  # noqa: F811
    """Given as an argument, the current stream is what it is without."""
    for name in sorted(CALLS):
        want = copies(CALLS[name](darb, pair[0]))
        assert same(flat(CALLS[name](darb, pair[0], stream=torch.cuda.current_stream())), want), name
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got = flat(CALLS[name](darb, pair[0], stream=st))
        st.synchronize()
        assert same(got, want), name
