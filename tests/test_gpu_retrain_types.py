"""The retraining chain, layer norm to optimizer, with hidden states of every type: fp32 as it is, 16
bits with the conversions where the product meets them (it takes fp32 or fp16 and gives fp32).

Each stage is compared with 64 bits from what the chain itself rounded to 16 bits (x, dx); the
bounds are those of one step of the retraining example, 1e-5 of the log probabilities' size,
relative to the largest gradient, and one rounding of dx."""
import numpy as np
import pytest

from tests._gpu import darb, dev, say, torch  # noqa: F401
from tests._train import ROUND, TYPES, wide

pytestmark = pytest.mark.gpu


def chain(d, plan, values, offsets, index, h, weight, bias, words, grad):
    x, mean, rstd = d.layer_norm(h, weight, bias)
    into = x.float() if x.dtype == torch.bfloat16 else x
    z = plan.spmm(values, offsets, into)
    r = d.token_logprobs(z, words, top=5)
    dz = d.token_logprobs_grad(z, words, r.lse, grad, out=z)
    dvalues, dx = plan.spmm_grad(index, values, into, dz)
    _, dw, db = d.layer_norm_grad(dx.to(h.dtype), h, mean, rstd, weight, need_x=False)
    return x, mean, rstd, r, dvalues, dx, dw, db


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_chain_of_each_type(darb, dtype):  # noqa: F811
    say(f"retraining chain: {dtype}")
    M, N, B = 257, 96, 50
    rng = np.random.default_rng(5)
    values_type = torch.float16 if dtype == "f16" else torch.float32
    plan = darb.Plan(M, N, np.full(M, 0.25), 0.25, darb.ROUND_FLOOR, 4, 4).upload()
    v, o = plan.encode(dev((rng.standard_normal((M, N)) * 0.3).astype(np.float32)))
    v = v.to(values_type)
    h = dev(rng.standard_normal((N, B)).astype(np.float32)).to(TYPES[dtype])
    weight = dev((1 + 0.2 * rng.standard_normal(N)).astype(np.float32))
    bias = dev((0.2 * rng.standard_normal(N)).astype(np.float32))
    words = torch.from_numpy(rng.integers(0, M, B)).cuda()
    grad = torch.full((B,), -1.0, device="cuda")
    x, mean, rstd, r, dv, dx, dw, db = chain(darb, plan, v, o, plan.transpose(o), h, weight, bias, words, grad)
    assert x.dtype == h.dtype and dv.dtype == dx.dtype == dw.dtype == torch.float32
    # the chain in 64 bits
    W, x64 = wide(plan.decode(v.float(), o)), wide(x)
    t = words.cpu().numpy()
    z = W @ x64
    lse = np.log(np.exp(z - z.max(0)).sum(0)) + z.max(0)
    logp = z[t, np.arange(B)] - lse
    dz = np.exp(z - lse) - (np.arange(M)[:, None] == t)
    size = 1e-5 * max(1.0, np.abs(logp).max())
    assert np.abs(wide(r.logprob) - logp).max() <= 2 * size
    got = wide(plan.decode(dv, o))
    at = wide(plan.decode(torch.ones_like(dv), o)) != 0
    full = (dz @ x64.T) * at
    assert np.abs(got - full).max() <= 4 * size * np.abs(full).max()
    want = W.T @ dz
    assert np.abs(wide(dx) - want).max() <= 4 * size * np.abs(want).max()
    # the layer norm's gradients, from dx before its rounding
    xh = (wide(h) - wide(mean)) * wide(rstd)
    rel, small = ROUND[dtype]
    for g, terms in ((dw, want * xh), (db, want)):
        slack = (rel * np.abs(terms) + small * np.maximum(np.abs(xh), 1)).sum(1)
        full = terms.sum(1)
        assert (np.abs(wide(g) - full) <= slack + 4 * size * np.abs(full).max() + 1e-12).all()
    # and a step on them, masters where values are of 16 bits
    opt = darb.AdamW([v, weight, bias], masters=True, state_bits=8)
    before = v.clone()
    opt.step([dv, dw, db])
    assert not torch.equal(v, before)
