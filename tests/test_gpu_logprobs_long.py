"""Log probabilities where the tokens take more than one launch."""
import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_tokens_than_a_launch_takes(darb, dtype):  # noqa: F811
    """Feature-major, 2^15 tiles of 64 tokens and some, and 2^20 tokens to a joining launch."""
    V, B = 3, (1 << 21) + 77
    say(f"log probabilities: {V} x {B} {dtype}")
    rng = torch.Generator(device="cuda").manual_seed(3)
    z = (torch.randn((V, B), device="cuda", generator=rng) * 3).to(dtype)
    t = torch.randint(0, V, (B,), device="cuda", generator=rng)
    g = torch.randn(B, device="cuda", generator=rng)
    r = darb.token_logprobs(z, t, top=2)
    logp = torch.log_softmax(z.double(), 0)
    # a few terms' roundings of 2^-23, of numbers below some 20
    bound = 1e-5
    assert bool(((r.logprob - logp.gather(0, t[None])[0]).abs() <= bound).all())
    assert bool(((r.lse - z.double().logsumexp(0)).abs() <= bound).all())
    H = -(logp.exp() * logp).sum(0)
    assert bool(((r.entropy - H).abs() <= 2 * bound * (1 + H)).all())
    order = torch.sort(z.float(), dim=0, descending=True, stable=True).indices[:2].t()
    assert torch.equal(r.top_index, order)
    dz = darb.token_logprobs_grad(z, t, r.lse, g)
    p = logp.exp()
    hit = torch.zeros_like(p).scatter_(0, t[None], 1.0)
    want = g.double() * (hit - p)
    off = 0.0 if dtype == torch.float32 else 2.0 ** -8
    assert bool(((dz - want).abs() <= g.abs() * bound * (hit + p) + off * want.abs() + 1e-30).all())
