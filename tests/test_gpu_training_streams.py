"""The evaluation and retraining calls on a given stream, beside work that waits on the current one:
no call's memory is another's.

The two streams get different inputs, the given one never waits for the current one, and every
buffer is of one size in both, so that a block handed out too early changes results."""
import numpy as np
import pytest

from tests._gpu import darb, dev, say, torch  # noqa: F401
from tests._streams import Busy, copies, flat, same, without_native
from tests._train import place

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def busy(darb):  # noqa: F811
    return Busy()


def inputs(d, seed):
    rng = np.random.default_rng(seed)
    M, N, B = 300, 260, 70
    b = np.random.default_rng(0).choice([4, 16], size=M)          # one pattern of sizes
    plan = d.Plan(M, N, 1.0 / b, 0.1, 0, 4, 16).upload()
    v, o = plan.encode(dev(rng.standard_normal((M, N)).astype(np.float32)))
    f = dict(plan=plan, v=v, o=o, X=dev(rng.standard_normal((N, B)).astype(np.float32)),
             dY=dev(rng.standard_normal((M, B)).astype(np.float32)),
             t=torch.from_numpy(rng.integers(0, M, B)).cuda(), index=plan.transpose(o),
             g=dev(rng.standard_normal(B).astype(np.float32)), w=dev(rng.standard_normal(M).astype(np.float32)))
    f["z"] = place(rng.standard_normal((M, B)), "features", "f32")
    f["dz"] = place(rng.standard_normal((M, B)), "features", "f32")
    f["h"] = place(rng.standard_normal((M, B)), "tokens", "bf16")
    f["r"], f["n"] = d.token_logprobs(f["z"], f["t"]), d.layer_norm(f["z"])
    # a dY large enough for the product's gradients to use a workspace
    f["X2"] = dev(rng.standard_normal((N, 2700)).astype(np.float32))
    f["dY2"] = dev(rng.standard_normal((M, 2700)).astype(np.float32))
    f["opt"] = d.AdamW([torch.zeros(5000, device="cuda"), torch.zeros(333, device="cuda")], state_bits=8)
    f["opt"].step([dev(rng.standard_normal(n).astype(np.float32)) for n in (5000, 333)])
    return f


def index_of(plan, index):
    """What a column index holds: the columns' starts and the weights (not the padding between)."""
    entries = ((plan.N + 1) * 4 + 255) // 256 * 256
    return index[:(plan.N + 1) * 4], index[entries:entries + plan.nnz * 8]


CALLS = {
    "token_logprobs": lambda d, f, **k: d.token_logprobs(f["z"], f["t"], top=3, **k),
    "token_logprobs_grad": lambda d, f, **k: d.token_logprobs_grad(f["z"], f["t"], f["r"].lse, f["g"], **k),
    "layer_norm": lambda d, f, **k: d.layer_norm(f["h"], f["w"], **k),
    "layer_norm_grad": lambda d, f, **k: d.layer_norm_grad(f["dz"], f["z"], f["n"][1], f["n"][2], f["w"], **k),
    "transpose": lambda d, f, **k: index_of(f["plan"], f["plan"].transpose(f["o"], **k)),
    "spmm_grad": lambda d, f, **k: f["plan"].spmm_grad(f["index"], f["v"], f["X"], f["dY"], **k),
    "spmm_grad split": lambda d, f, **k: f["plan"].spmm_grad(f["index"], f["v"], f["X2"], f["dY2"], **k),
    "moments": lambda d, f, **k: f["opt"].moments(**k),
}


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


def test_a_stream_that_torch_does_not_know(darb, pair):  # noqa: F811
    """Any object with a stream's handle will do."""
    class Handle:
        def __init__(self, s):
            self.cuda_stream = s.cuda_stream
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for name in sorted(CALLS):
        want = copies(CALLS[name](darb, pair[0]))
        got = CALLS[name](darb, pair[0], stream=Handle(st))
        torch.cuda.synchronize()
        assert same(flat(got), want), name


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_made_for_a_given_stream(darb, busy, bits):  # noqa: F811
    """The masters and the first states are there when the given stream's first step reads them."""
    say(f"adamw made for a given stream: {bits} bits")
    sizes = [70000, 257, 1]
    start = [torch.randn(n, device="cuda").half() for n in sizes]
    grads = [torch.randn(n, device="cuda") for n in sizes]
    p = [t.clone() for t in start]
    want = darb.AdamW(p, masters=True, state_bits=bits)
    want.step(grads)
    want = copies([p, want.masters, want.moments()])
    p = [t.clone() for t in start]
    st = torch.cuda.Stream()
    # memory that is handed out again holds no zeros
    for n in sizes:
        for kind in (torch.float32, torch.uint8):
            junk = [torch.full((n,), 77, dtype=kind, device="cuda") for _ in range(4)]
            del junk
    torch.cuda.synchronize()
    busy.queue()
    opt = darb.AdamW(p, masters=True, state_bits=bits, stream=st)
    opt.step(grads, stream=st)
    got = flat([p, opt.masters, opt.moments(stream=st)])
    torch.cuda.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("given", [True, False])
def test_adamw_dropped_before_its_step_is_done(darb, busy, given):  # noqa: F811
    """The step's table, states and masters are not handed out while its stream still needs them."""
    say(f"adamw dropped: stream {'given' if given else 'current'}")
    sizes = [70000, 257]
    start = [torch.randn(n, device="cuda").half() for n in sizes]
    grads = [torch.randn(n, device="cuda") for n in sizes]
    p = [t.clone() for t in start]
    darb.AdamW(p, masters=True, lr=0.1).step(grads)
    want = copies(p)
    p = [t.clone() for t in start]
    opt = darb.AdamW(p, masters=True, lr=0.1)
    held = [opt.workspace, *opt.masters, *flat(opt.state_tensors)]
    ranges = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in held]
    like = [(t.shape, t.dtype) for t in held]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        busy.queue()
        if not given:
            opt.step(grads)
    if given:
        opt.step(grads, stream=st)
    del opt, held
    new = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in like * 3]
    for t in new:
        begin, end = t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()
        assert all(end <= a or b <= begin for a, b in ranges)
        t.fill_(85)
    torch.cuda.synchronize()
    assert same(p, want)


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
