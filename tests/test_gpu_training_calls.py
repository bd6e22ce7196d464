"""The native call module against the Python code of the evaluation and retraining calls: the
same results bit for bit, in both memory orders, on a given stream and the current one."""
import numpy as np
import pytest

from tests._gpu import darb, dev, say, torch  # noqa: F401
from tests._train import place

pytestmark = pytest.mark.gpu


class Plain(torch.Tensor):
    """A tensor subclass: the native module leaves it to the Python code."""


def plain(t):
    return t.as_subclass(Plain)


def flat(r):
    return [None if t is None else t.as_subclass(torch.Tensor) for t in (r if isinstance(r, tuple) else (r,))]


@pytest.fixture(scope="module")
def f(darb):  # noqa: F811
    rng = np.random.default_rng(3)
    M, N, B = 90, 133, 21
    b = rng.choice([4, 16], size=M)
    plan = darb.Plan(M, N, 1.0 / b, 0.1, 0, 4, 16).upload()
    v, o = plan.encode(dev(rng.standard_normal((M, N)).astype(np.float32)))
    d = dict(plan=plan, v=v, o=o, index=plan.transpose(o), X=dev(rng.standard_normal((N, B)).astype(np.float32)),
             dY=dev(rng.standard_normal((M, B)).astype(np.float32)), t=torch.from_numpy(rng.integers(0, M, B)).cuda(),
             g=dev(rng.standard_normal(B).astype(np.float32)), w=dev(rng.standard_normal(M).astype(np.float32)))
    for order in ("features", "tokens"):
        d[order] = place(rng.standard_normal((M, B)), order, "bf16")
        d["dy " + order] = place(rng.standard_normal((M, B)), order, "bf16")
    d["r"] = darb.token_logprobs(d["features"], d["t"], top=3)
    d["n"] = darb.layer_norm(d["features"])
    return d


CALLS = {
    "token_logprobs": lambda d, f, o, w, **k: d.token_logprobs(w(f[o]), f["t"], top=3, **k),
    "token_logprobs bare": lambda d, f, o, w, **k: d.token_logprobs(w(f[o]), **k),
    "token_logprobs_grad": lambda d, f, o, w, **k: d.token_logprobs_grad(w(f[o]), f["t"], f["r"].lse, f["g"],
                                                                        f["r"].entropy, f["g"], **k),
    "layer_norm": lambda d, f, o, w, **k: d.layer_norm(w(f[o]), f["w"], None, **k),
    "layer_norm_grad": lambda d, f, o, w, **k: d.layer_norm_grad(w(f["dy " + o]), f[o], f["n"][1], f["n"][2],
                                                                f["w"], **k),
    "spmm_grad": lambda d, f, o, w, **k: f["plan"].spmm_grad(f["index"], w(f["v"]), f["X"], f["dY"], **k),
}


@pytest.mark.parametrize("order", ["features", "tokens"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_native_call_equals_python_path(darb, f, name, order):  # noqa: F811
    say(f"native call: {name} {order}")
    want = flat(CALLS[name](darb, f, order, plain))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    results = [CALLS[name](darb, f, order, lambda t: t), CALLS[name](darb, f, order, lambda t: t, stream=st)]
    with torch.cuda.stream(st):
        results.append(CALLS[name](darb, f, order, lambda t: t))
    st.synchronize()
    for got in results:
        got = flat(got)
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert a is None and b is None or (a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a, b))


def test_native_outputs_given(darb, f):  # noqa: F811
    x = f["tokens"]
    y, mean, rstd = torch.empty_like(x), torch.empty(21, device="cuda"), torch.empty(21, device="cuda")
    got = darb.layer_norm(x, f["w"], y=y, mean=mean, rstd=rstd)
    assert got[0] is y and got[1] is mean and got[2] is rstd
    out = torch.empty_like(x)
    assert darb.token_logprobs_grad(x, f["t"], f["r"].lse, f["g"], out=out) is out


def test_native_adamw_equals_python_path(darb):  # noqa: F811
    p = [torch.randn(n, device="cuda") for n in (5, 300, 1)]
    q = [t.clone() for t in p]
    a, b = darb.AdamW(p, state_bits=8), darb.AdamW(q, state_bits=8)
    scale = torch.tensor([0.25], device="cuda")
    for k in range(3):
        g = [torch.randn_like(t).bfloat16() for t in p]
        g[2] = None if k == 1 else g[2]
        a.step(g, grad_scale=scale)
        b.step([None if t is None else plain(t) for t in g], grad_scale=scale)
    assert a.steps == b.steps == 3
    m, n = a.moments(), b.moments(out=tuple([plain(torch.empty_like(t)) for t in q] for _ in range(2)))
    for x, y in zip(p + m[0] + m[1], q + n[0] + n[1]):
        assert torch.equal(x, y.as_subclass(torch.Tensor))


def test_one_token_goes_on_into_a_product(darb, f):  # noqa: F811
    """A single token leaves the memory order open: the norm's output and the gradients' are
    contiguous, as the products take them."""
    for wrap in (plain, lambda t: t):
        h = f["X"][:, :1].contiguous()
        y, mean, rstd = darb.layer_norm(wrap(h))
        f["plan"].spmm(f["v"], f["o"], y)
        r = darb.token_logprobs(y)
        dz = darb.token_logprobs_grad(wrap(y), None, r.lse, r.logprob)
        dx = darb.layer_norm_grad(wrap(y), h, mean, rstd)[0]
        for t in (y, dz, dx):
            assert t.is_contiguous() and t.stride(1) == 1
