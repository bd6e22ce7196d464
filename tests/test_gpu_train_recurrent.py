"""A recurrent language model's training step, all calls together, against 64-bit arithmetic; and what
the package's functions refuse."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb  # noqa: E402,F401

pytestmark = pytest.mark.gpu

H, V, T, BATCH = 48, 90, 12, 8
COLUMNS = T * BATCH


class Model:
    """Columns x of embeddings, a gated recurrence fed by two dense matrices, layer norm, and a DARB output
    layer."""

    def __init__(self, darb, kind=torch.float32):
        r = np.random.default_rng(3)
        f = lambda *s: torch.from_numpy(r.normal(size=s) * 0.3).float().cuda()       # noqa: E731
        self.x = f(H, COLUMNS)
        self.Wg, self.Wx = f(H, H), f(H, H)
        self.weight, self.bias = 1 + f(H), f(H)
        W = f(V, H)
        counts = darb.prune_counts(W, V * H // 4)
        self.plan = darb.Plan.from_device_counts(H, counts, V * H // 4, darb.ROUND_FLOOR, 1, 16)
        self.values, self.offsets = self.plan.encode(W)
        self.index = self.plan.transpose(self.offsets)
        self.targets = torch.from_numpy(r.integers(0, V, COLUMNS)).cuda()
        self.targets[::7] = -1
        self.starts = torch.from_numpy(r.random(COLUMNS) < 0.1).cuda()
        self.old, self.ref, self.adv = (torch.from_numpy(r.normal(size=COLUMNS) * s + m).float().cuda()
                                        for s, m in ((0.2, -4.5), (0.3, -4.5), (1.0, 0.0)))
        self.w = torch.from_numpy(np.where(r.random(COLUMNS) < 0.2, 0, 1 / COLUMNS)).float().cuda()
        self.w[self.targets < 0] = 0
        self.darb = darb

    def forward(self):
        d = self.darb
        self.z, self.u = self.Wg @ self.x, self.Wx @ self.x
        self.h, _ = d.gated_recurrence(self.z, self.u, batch=BATCH, resets=self.starts)
        self.n, self.mean, self.rstd = d.layer_norm(self.h, self.weight, self.bias)
        self.y = self.plan.spmm(self.values, self.offsets, self.n)
        return d.token_logprobs(self.y, self.targets)

    def backward(self, r, grad, grad_entropy=None):
        d = self.darb
        dy = d.token_logprobs_grad(self.y, self.targets, r.lse, grad, r.entropy if grad_entropy is not None else None,
                                   grad_entropy)
        dv, dn = self.plan.spmm_grad(self.index, self.values, self.n, dy)
        dh, dw, db = d.layer_norm_grad(dn, self.h, self.mean, self.rstd, self.weight)
        dz, du, _ = d.gated_recurrence_grad(dh, self.z, self.u, self.h, batch=BATCH, resets=self.starts)
        return dz @ self.x.t(), du @ self.x.t(), dv, dw, db


def in_64_bits(m, kind):
    """(loss, gradients) through automatic differentiation, from the same numbers."""
    leaf = lambda t: t.double().cpu().requires_grad_()                               # noqa: E731
    Wg, Wx, v, w, b = (leaf(t) for t in (m.Wg, m.Wx, m.values, m.weight, m.bias))
    x, starts = m.x.double().cpu(), m.starts.cpu().view(T, BATCH)
    f, u = torch.sigmoid(Wg @ x).view(H, T, BATCH), (Wx @ x).view(H, T, BATCH)
    state, hs = torch.zeros(H, BATCH, dtype=torch.float64), []
    for t in range(T):
        state = torch.where(starts[t], torch.zeros_like(state), state)
        state = f[:, t] * state + (1 - f[:, t]) * u[:, t]
        hs.append(state)
    h = torch.stack(hs, 1).reshape(H, COLUMNS)
    n = (h - h.mean(0)) / torch.sqrt(h.var(0, correction=0) + 1e-5) * w[:, None] + b[:, None]
    W = m.plan.decode(torch.arange(1, m.plan.nnz + 1, device="cuda").float(), m.offsets).long().cpu()
    dense = torch.zeros(V, H, dtype=torch.float64)
    dense = torch.where(W > 0, v[(W - 1).clamp(min=0)], dense)
    y = torch.log_softmax(dense @ n, 0)
    t = m.targets.cpu()
    lp = torch.where(t >= 0, y.gather(0, t.clamp(min=0)[None])[0], torch.zeros(COLUMNS, dtype=torch.float64))
    c = lambda a: a.double().cpu()                                                   # noqa: E731
    if kind == "policy":
        ratio = torch.exp(lp - c(m.old))
        A = c(m.adv)
        q = c(m.ref) - lp
        L = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A) + 0.05 * (torch.exp(q) - 1 - q) + \
            0.01 * (y.exp() * y).sum(0)
        loss = (c(m.w) * L).sum()
    else:
        d = torch.where(t >= 0, lp - c(m.ref), torch.zeros_like(lp)).view(T, BATCH).sum(0)
        margin = 0.3 * (d[:BATCH // 2] - d[BATCH // 2:])
        loss = -torch.nn.functional.logsigmoid(margin).mean()
    return float(loss), torch.autograd.grad(loss, (Wg, Wx, v, w, b))


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_one_step(darb, kind):
    m = Model(darb)
    r = m.forward()
    if kind == "policy":
        lo = darb.policy_loss(r.logprob, m.old, m.adv, weight=m.w, clip=0.2, ref_logprob=m.ref, kl_coef=0.05,
                              entropy=r.entropy, entropy_coef=0.01)
        grads = m.backward(r, lo.grad_logprob, lo.grad_entropy)
    else:
        m.ref[m.targets < 0] = 0
        lo = darb.preference_loss(r.logprob, m.ref, batch=BATCH, beta=0.3)
        grads = m.backward(r, lo.grad_logprob)
    want, gw = in_64_bits(m, kind)
    # a few hundred fp32 roundings on the way, through 12 steps and a norm: 1e-5 of the norms
    assert abs(float(lo.loss) - want) <= 1e-5 * max(1.0, abs(want))
    for name, g, e in zip(("Wg", "Wx", "values", "weight", "bias"), grads, gw):
        off, size = float((g.double().cpu() - e).norm()), float(e.norm())
        assert size > 0 and off <= 1e-5 * size * 4, (name, off, size)


def test_training_runs(darb):
    """Steps of both optimizers over the model's tensors change what they should and stay finite."""
    m = Model(darb)
    dense, rest = [m.Wg, m.Wx], [m.values, m.weight, m.bias]
    before = [t.clone() for t in dense + rest]
    muon, adam = darb.Muon(dense, lr=0.02), darb.AdamW(rest, lr=1e-3)
    for _ in range(4):
        r = m.forward()
        lo = darb.policy_loss(r.logprob, m.old, m.adv, weight=m.w)
        grads = m.backward(r, lo.grad_logprob)
        muon.step(grads[:2])
        adam.step(list(grads[2:]))
    for a, b in zip(before, dense + rest):
        assert torch.isfinite(b).all() and not torch.equal(a, b)


def test_step_by_step_is_the_sequence(darb):
    """Generating one step at a time gives the sequence's states."""
    torch.manual_seed(1)
    for kind, tol in ((torch.float32, 40 * 2.0 ** -24), (torch.bfloat16, 2.0 ** -7)):
        z, x = (torch.randn(64, 40 * 3, device="cuda").to(kind) for _ in range(2))
        h, last = darb.gated_recurrence(z, x, batch=3)
        state = torch.zeros(64, 3, device="cuda")
        for t in range(40):
            c = slice(3 * t, 3 * t + 3)
            out, same = darb.gated_recurrence(z[:, c].contiguous(), x[:, c].contiguous(), batch=3, h0=state, h_last=state)
            assert same is state
            # two roundings a step of values below 5, carried on by f < 1
            assert float((out.float() - h[:, c].float()).abs().max()) <= 5 * tol
        assert float((state - last).abs().max()) <= 5 * 40 * 2.0 ** -24


NAMES = ("gated_recurrence", "gated_recurrence_grad", "policy_loss", "preference_loss")


def test_native_and_python_calls_agree(darb, monkeypatch):
    torch.manual_seed(0)
    z, x, dh = (torch.randn(20, 24, device="cuda") for _ in range(3))
    s = torch.randn(20, 3, device="cuda")
    lp, old, adv, w, rf, en = (torch.randn(24, device="cuda") for _ in range(6))
    starts = torch.tensor([0, 5, 20], device="cuda")
    cuts = torch.rand(24, device="cuda") < 0.3

    def every(stream=None):
        h = darb.gated_recurrence(z, x, batch=3, h0=s, resets=cuts, stream=stream)
        return [*h, *darb.gated_recurrence_grad(dh, z, x, h[0], batch=3, h0=s, resets=cuts, dh_last=s, stream=stream),
                *darb.gated_recurrence(z.t().contiguous().t(), x.t().contiguous().t(), batch=8, form="linear"),
                *darb.policy_loss(lp, old, adv, stream=stream)[:4],
                *darb.policy_loss(lp, old, adv, w, (0.1, 0.3), rf, 0.1, en, 0.2),
                *darb.preference_loss(lp, rf, batch=6), *darb.preference_loss(lp, starts=starts, weight=w[:1].clone())]
    native = [t.clone() for t in every()]
    for name in NAMES:
        monkeypatch.setattr(darb._native, name, lambda *a: None)
    for stream in (None, torch.cuda.Stream()):
        torch.cuda.synchronize()
        got = every(stream)
        torch.cuda.synchronize()
        assert len(got) == len(native)
        for a, b in zip(got, native):
            assert a.stride() == b.stride() and torch.equal(a, b)


def test_refusals(darb):
    x, v = torch.zeros(4, 6, device="cuda"), torch.zeros(6, device="cuda")
    s = torch.zeros(4, 3, device="cuda")
    starts = torch.tensor([0, 3, 6], device="cuda")
    bad = [
        (ValueError, lambda: darb.gated_recurrence(x, x, batch=4)),
        (ValueError, lambda: darb.gated_recurrence(x, x, batch=0)),
        (ValueError, lambda: darb.gated_recurrence(x, x, form="no")),
        (TypeError, lambda: darb.gated_recurrence(x, x.half())),
        (TypeError, lambda: darb.gated_recurrence(x.double(), x.double())),
        (ValueError, lambda: darb.gated_recurrence(x, x[:, :4])),
        (ValueError, lambda: darb.gated_recurrence(x, x, batch=3, h0=s[:, :2])),
        (ValueError, lambda: darb.gated_recurrence(x, x, batch=3, h0=s.half())),
        (ValueError, lambda: darb.gated_recurrence(x, x, resets=v[:5].bool())),
        (TypeError, lambda: darb.gated_recurrence(x, x, resets=v)),
        (ValueError, lambda: darb.gated_recurrence(x, x, resets=v.bool().cpu())),
        (darb.DarbError, lambda: darb.gated_recurrence(x, x.t().contiguous().t())),
        (ValueError, lambda: darb.gated_recurrence_grad(x, x, None, x)),
        (darb.DarbError, lambda: darb.gated_recurrence_grad(x, x, x, x, dx=x)),
        (ValueError, lambda: darb.gated_recurrence_grad(x, x, x, x[:3])),
        (ValueError, lambda: darb.policy_loss(v, v, v[:5])),
        (ValueError, lambda: darb.policy_loss(v, v, None)),
        (ValueError, lambda: darb.policy_loss(v, v, v, weight=v[::2])),
        (TypeError, lambda: darb.policy_loss(v.half(), v, v)),
        (darb.DarbError, lambda: darb.policy_loss(v, v, v, kl_coef=0.1)),
        (darb.DarbError, lambda: darb.policy_loss(v, v, v, clip=-1)),
        (ValueError, lambda: darb.preference_loss(v)),
        (ValueError, lambda: darb.preference_loss(v, batch=2, starts=starts)),
        (ValueError, lambda: darb.preference_loss(v, batch=3)),
        (ValueError, lambda: darb.preference_loss(v, batch=4)),
        (ValueError, lambda: darb.preference_loss(v, starts=starts[:2])),
        (TypeError, lambda: darb.preference_loss(v, starts=starts.int())),
        (ValueError, lambda: darb.preference_loss(v, batch=2, weight=v)),
        (darb.DarbError, lambda: darb.preference_loss(v, batch=2, label_smoothing=1.0)),
        (TypeError, lambda: darb.orthogonalize(x.double())),
        (ValueError, lambda: darb.orthogonalize(v)),
        (ValueError, lambda: darb.orthogonalize(x[:0])),
        (ValueError, lambda: darb.orthogonalize(torch.zeros(4, 12, device="cuda")[::1, ::2][:, :5].t()[::2])),
        (ValueError, lambda: darb.orthogonalize(x, out=x.half())),
        (ValueError, lambda: darb.orthogonalize(x.expand(3, 4, 6), out=x.expand(3, 4, 6))),
        (darb.DarbError, lambda: darb.orthogonalize(x, steps=0)),
        (darb.DarbError, lambda: darb.orthogonalize(x, eps=0)),
        (ValueError, lambda: darb.Muon([v])),
        (ValueError, lambda: darb.Muon([x.t()])),
        (ValueError, lambda: darb.Muon([x], masters=[s])),
        (ValueError, lambda: darb.Muon([x], state=[x, x])),
        (ValueError, lambda: darb.Muon([x]).step([x, x])),
        (ValueError, lambda: darb.Muon([x]).step([s])),
        (ValueError, lambda: darb.Muon([x]).step([x.cpu()])),
        (TypeError, lambda: darb.Muon([x]).step([x.double()]))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("not refused:", i)
