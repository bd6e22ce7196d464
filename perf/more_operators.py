"""Performance cases of the operators that train a recurrent language model around its DARB
layers: a gated linear recurrence over sequences with its gradients, the losses of preference
and policy training over token log probabilities with their gradients, and the orthogonalised
update of weight matrices.

Activations are [features x columns], column t * batch + n holding step t of sequence n, as the
LSTM layer's sequences are: feature-major ("features"), or token-major ("tokens"), which reaches
the calls as a transposed view.  Token log probabilities are flat, in that order of columns, or
packed sequence after sequence.

``own`` false computes each operator in elementary torch operations, in 32 bits (long sums in
64); true calls the framework.  Sizes are those of the workloads (1024-wide LSTM with 200 steps
of 32, the 4096 x 9216 head, the 1500-wide language model of the paper) and generic ones around
them.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
CLIP_LOW, CLIP_HIGH, KL, ENTROPY = 0.2, 0.28, 0.05, 0.01
BETA, SMOOTHING = 0.1, 0.05
LR, MOMENTUM, DECAY, NS_EPS, NS_STEPS = 0.02, 0.95, 0.1, 1e-7, 5
NS = (3.4445, -4.7750, 2.0315)       # the quintic's coefficients


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------

def _recurrence(op, H, T, batch, dtype, order, form="gate", resets=False):
    return dict(op=op, H=H, T=T, batch=batch, dtype=dtype, order=order, form=form, resets=resets)


def _policy(tokens, reference, entropy):
    return dict(op="policy", tokens=tokens, reference=reference, entropy=entropy)


def _preference(pairs, length, packed):
    return dict(op="preference", pairs=pairs, length=length, packed=packed)


def _orthogonalize(count, m, n, dtype):
    return dict(op="orthogonalize", count=count, m=m, n=n, dtype=dtype)


def _muon(layers, width, inner, dtype, gdtype, masters):
    return dict(op="muon", layers=layers, width=width, inner=inner, dtype=dtype, gdtype=gdtype,
                masters=masters)


def listed():
    cases = {
        # one generated token of 32 sequences: the layer's step in serving (latency)
        "recurrence_step": _recurrence("recurrence", 1024, 1, 32, "f32", "features"),
        # a layer over the sequences of the 1024-wide LSTM, straight from the product's output
        "recurrence_seq": _recurrence("recurrence", 1024, 200, 32, "f32", "features"),
        # its gradients
        "recurrence_grad_seq": _recurrence("recurrence_grad", 1024, 200, 32, "f32", "features"),
        # packed texts in one long sequence, token-major bf16: few series, much time
        "recurrence_long_bf16": _recurrence("recurrence", 1024, 65536, 1, "bf16", "tokens",
                                            resets=True),
        # gradients of the plain linear form, one feature-major sequence of odd length, fp16
        "recurrence_grad_odd_f16": _recurrence("recurrence_grad", 1500, 2999, 1, "f16",
                                               "features", "linear"),
        # the policy loss of 35 steps of a batch of 20 (latency)
        "policy_lm": _policy(700, True, False),
        # a large rollout's, with the entropy's part, an odd number of tokens
        "policy_large": _policy(1_000_003, True, True),
        # preferences of 64 pairs, padded to 512 steps
        "preference_padded": _preference(64, 512, False),
        # preferences of many packed pairs of unlike lengths
        "preference_packed": _preference(1500, 1400, True),
        # eight small bf16 matrices at once
        "orthogonalize_small_bf16": _orthogonalize(8, 256, 1024, "bf16"),
        # the dense 4096 x 9216 head in fp32
        "orthogonalize_fc": _orthogonalize(1, 4096, 9216, "f32"),
        # a step over the matrices of a 1500-wide language model, fp32 masters of bf16
        "muon_lm": _muon(2, 1500, 6000, "bf16", "bf16", True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice([1, 1, 4, 16, 64])     # most sizes are multiples of something
    return max(lo, min(hi, v // step * step))


def draw(rng):
    kind = rng.choice(["recurrence", "recurrence_grad", "policy", "preference", "orthogonalize",
                       "muon"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind.startswith("recurrence"):
        H = _log_int(rng, 16, 4096)
        batch = rng.choice([1, 1, _log_int(rng, 2, 256), 20, 32])
        T = _log_int(rng, 1, max(1, min(65536, 12_000_000 // (H * batch))))
        return _recurrence(kind, H, T, batch, dtype, rng.choice(["features", "tokens"]),
                           rng.choice(["gate", "linear"]), rng.random() < 0.4)
    if kind == "policy":
        return _policy(_log_int(rng, 1, 1_000_000), rng.random() < 0.7, rng.random() < 0.5)
    if kind == "preference":
        pairs = _log_int(rng, 1, 4000)
        return _preference(pairs, _log_int(rng, 1, max(1, min(4096, 2_000_000 // pairs))),
                           rng.random() < 0.5)
    if kind == "orthogonalize":
        m = _log_int(rng, 32, 4096)
        n = _log_int(rng, 32, 6144)
        count = _log_int(rng, 1, max(1, min(16, 20_000_000_000 // (m * n * min(m, n)))))
        return _orthogonalize(count, m, n, dtype)
    width = _log_int(rng, 64, 1500)
    return _muon(_log_int(rng, 1, 4), width, _log_int(rng, width, 4 * width), dtype,
                 rng.choice(["f32", dtype]), dtype != "f32" and rng.random() < 0.6)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _ordered(t, order):
    """A [features, columns] tensor's values in the memory order asked for."""
    return t.contiguous() if order == "features" else t.t().contiguous().t()


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op.startswith("recurrence"):
        return _prepare_recurrence(case, g)
    if op == "policy":
        return _prepare_policy(case, g)
    if op == "preference":
        return _prepare_preference(case, g)
    if op == "orthogonalize":
        shape = (case["count"], case["m"], case["n"])
        return dict(case=case, G=_gradient(g, *shape).to(TYPES[case["dtype"]]))
    return _prepare_muon(case, g)


def _prepare_recurrence(case, g):
    H, T, n = case["H"], case["T"], case["batch"]
    kind, order = TYPES[case["dtype"]], case["order"]

    def normal(spread=1.0, shift=0.0):
        return torch.randn(H, T * n, generator=g, device=DEV) * spread + shift

    gate, x = normal(1.5, 1.0), normal()
    if case["form"] == "linear":             # decays, and inputs of the same scale
        gate = torch.sigmoid(gate + 1)
        x = x * torch.sqrt(1 - gate * gate)
    s = dict(case=case, gate=_ordered(gate.to(kind), order), x=_ordered(x.to(kind), order),
             h0=_ordered(torch.randn(H, n, generator=g, device=DEV), order), resets=None)
    if case["resets"]:                       # a packed text starts every few hundred steps
        s["resets"] = torch.rand(T * n, generator=g, device=DEV) < 1 / 300
    if case["op"] == "recurrence_grad":
        s["h"] = _plain_recurrence(s)["h"]
        s["dh"] = _ordered(normal(0.1).to(kind), order)
        s["dh_last"] = _ordered(0.1 * torch.randn(H, n, generator=g, device=DEV), order)
    return s


def _prepare_policy(case, g):
    n = case["tokens"]
    normal = lambda: torch.randn(n, generator=g, device=DEV)                     # noqa: E731
    lp = -2 * torch.rand(n, generator=g, device=DEV).log().abs()
    s = dict(case=case, lp=lp, old=lp + 0.15 * normal(), advantage=normal(),
             reference=lp + 0.3 * normal() if case["reference"] else None, entropy=None)
    if case["entropy"]:
        s["entropy"] = 3 * torch.rand(n, generator=g, device=DEV)
    live = torch.rand(n, generator=g, device=DEV) > 1 / 8               # the others are prompts
    live[0] = True
    s["weight"] = live / live.sum()
    return s


def _prepare_preference(case, g):
    S, L = 2 * case["pairs"], case["length"]
    s = dict(case=case, starts=None)
    if case["packed"]:                       # half of the length on average, some of 0
        n = max(1, S * L // 2)
        cuts = torch.randint(0, n + 1, (S - 1,), generator=g, device=DEV).sort().values
        s["starts"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)])
        live = torch.ones(n, device=DEV)
    else:
        n = S * L
        lengths = (torch.rand(S, generator=g, device=DEV) * L).long() + 1
        live = (torch.arange(L, device=DEV)[:, None] < lengths).float().view(-1)
    lp = -2 * torch.rand(n, generator=g, device=DEV).log().abs()
    s["lp"] = live * lp                      # a padded place has log probability 0 twice
    s["reference"] = live * (lp + 0.1 * torch.randn(n, generator=g, device=DEV))
    return s


def _gradient(g, count, m, n):
    """Gradients as they are met: a part of low rank over noise."""
    r = max(1, min(m, n) // 16)
    a = torch.randn(count, m, r, generator=g, device=DEV)
    b = torch.randn(count, r, n, generator=g, device=DEV)
    return 1e-3 * (torch.bmm(a, b) / math.sqrt(r) +
                   torch.randn(count, m, n, generator=g, device=DEV))


def _shapes(case):
    """The matrices of a model: square ones, and those into and out of a wider layer."""
    w, i = case["width"], case["inner"]
    return [shape for _ in range(case["layers"]) for shape in ((w, w), (w, w), (i, w), (w, i))]


def _prepare_muon(case, g):
    kind = TYPES[case["dtype"]]
    s = dict(case=case, p=[], g=[], m=[], master=[])
    for rows, cols in _shapes(case):
        w = 0.02 * torch.randn(rows, cols, generator=g, device=DEV)
        s["p"].append(w.to(kind))
        s["master"].append(w if case["masters"] else None)
        s["g"].append(_gradient(g, 1, rows, cols)[0].to(TYPES[case["gdtype"]]))
        s["m"].append(_gradient(g, 1, rows, cols)[0])
    if own:
        import paper_1911_08020_amd as darb
        s["optimizer"] = darb.Muon(s["p"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY,
                                   eps=NS_EPS, steps=NS_STEPS, state=s["m"],
                                   masters=s["master"] if case["masters"] else None)
    return s


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return PLAIN[state["case"]["op"]](state)


def _run_own(s):
    import paper_1911_08020_amd as darb
    c = s["case"]
    if c["op"] == "recurrence":
        h, last = darb.gated_recurrence(s["gate"], s["x"], batch=c["batch"], h0=s["h0"],
                                        resets=s["resets"], form=c["form"])
        return dict(h=h, last=last)
    if c["op"] == "recurrence_grad":
        dgate, dx, dh0 = darb.gated_recurrence_grad(
            s["dh"], s["gate"], s["x"], s["h"], batch=c["batch"], h0=s["h0"],
            resets=s["resets"], dh_last=s["dh_last"], form=c["form"])
        return dict(dgate=dgate, dx=dx, dh0=dh0)
    if c["op"] == "policy":
        r = darb.policy_loss(s["lp"], s["old"], s["advantage"], weight=s["weight"],
                             clip=(CLIP_LOW, CLIP_HIGH), ref_logprob=s["reference"],
                             kl_coef=KL if c["reference"] else 0.0, entropy=s["entropy"],
                             entropy_coef=ENTROPY if c["entropy"] else 0.0)
        out = dict(loss=r.loss, kl=r.kl, clipped=r.clipped, dlp=r.grad_logprob)
        if c["entropy"]:
            out["dentropy"] = r.grad_entropy
        return out
    if c["op"] == "preference":
        r = darb.preference_loss(s["lp"], s["reference"], starts=s["starts"],
                                 batch=None if c["packed"] else 2 * c["pairs"], beta=BETA,
                                 label_smoothing=SMOOTHING)
        return dict(loss=r.loss, margin=r.margin, dlp=r.grad_logprob)
    if c["op"] == "orthogonalize":
        return dict(O=darb.orthogonalize(s["G"], steps=NS_STEPS, eps=NS_EPS))
    s["optimizer"].step(s["g"])
    return _muon_outputs(s)


def _muon_outputs(s):
    out = dict(p=s["p"], m=s["m"])
    if s["case"]["masters"]:
        out["master"] = s["master"]
    return out


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------

def _steps_of(t, case):
    """[H, T * batch] as fp32 [T, H, batch]."""
    return t.float().view(case["H"], case["T"], case["batch"]).permute(1, 0, 2)


def _columns_of(t, case):
    return _ordered(t.permute(1, 0, 2).reshape(case["H"], -1).to(TYPES[case["dtype"]]),
                    case["order"])


def _scan(a, b):
    """y_t = a_t y_{t-1} + b_t over the first axis (y_{-1} = 0), by doubled strides."""
    T, d = a.shape[0], 1
    while d < T:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _decay_and_input(s):
    """f_t and what h_t takes from x_t, the state's share of f_t being 0 at a restart."""
    c = s["case"]
    z, x = _steps_of(s["gate"], c), _steps_of(s["x"], c)
    f, u = (torch.sigmoid(z), torch.sigmoid(-z)) if c["form"] == "gate" else (z, None)
    kept = f
    if s["resets"] is not None:
        kept = torch.where(s["resets"].view(c["T"], 1, c["batch"]), 0.0, f)
    return f, u, x, kept


def _plain_recurrence(s):
    c = s["case"]
    f, u, x, kept = _decay_and_input(s)
    b = x if u is None else u * x
    b = torch.cat([b[:1] + kept[:1] * s["h0"], b[1:]])
    h = _scan(kept, b)
    return dict(h=_columns_of(h, c), last=h[-1].contiguous())


def _plain_recurrence_grad(s):
    c = s["case"]
    f, u, x, kept = _decay_and_input(s)
    h, dh = _steps_of(s["h"], c), _steps_of(s["dh"], c)
    dh = torch.cat([dh[:-1], dh[-1:] + s["dh_last"]])
    # g_t = dh_t + kept_{t+1} g_{t+1}
    g = _scan(torch.cat([kept[1:], kept[:1] * 0]).flip(0), dh.flip(0)).flip(0)
    before = torch.cat([s["h0"][None], h[:-1]])
    if s["resets"] is not None:
        before = torch.where(s["resets"].view(c["T"], 1, c["batch"]), 0.0, before)
    dgate, dx = before * g, g
    if u is not None:
        dgate, dx = (before - x) * g * (f * u), u * g
    return dict(dgate=_columns_of(dgate, c), dx=_columns_of(dx, c), dh0=kept[0] * g[0])


def _plain_policy(s):
    lp, A, w = s["lp"], s["advantage"], s["weight"]
    # in 64 bits: which ratios are past a bound decides whole gradients
    ratio = torch.exp(lp.double() - s["old"].double())
    one, two = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    cut = two < one
    loss, d = -torch.minimum(one, two).float(), -torch.where(cut, 0.0, one).float()
    kl = torch.zeros_like(lp)
    if s["reference"] is not None:
        q = s["reference"] - lp
        kl = torch.expm1(q) - q
        loss = loss + KL * kl
        d = d - KL * torch.expm1(q)
    out = {}
    if s["entropy"] is not None:
        loss = loss - ENTROPY * s["entropy"]
        out["dentropy"] = -ENTROPY * w
    live = w != 0
    total = lambda v: torch.where(live, v * w, 0.0).double().sum().float()       # noqa: E731
    return dict(out, loss=total(loss), kl=total(kl), clipped=total(cut.float()),
                dlp=torch.where(live, d * w, 0.0))


def _plain_preference(s):
    P = s["case"]["pairs"]
    d = (s["lp"] - s["reference"]).double()
    if s["starts"] is None:
        sums = d.view(-1, 2 * P).sum(0)
    else:
        sums = torch.zeros(len(d) + 1, dtype=torch.float64, device=DEV)
        sums[1:] = torch.cumsum(d, 0)
        sums = sums[s["starts"][1:]] - sums[s["starts"][:-1]]
    margin = (BETA * (sums[:P] - sums[P:])).float()
    # - log sigma(m) = log(1 + e^-m)
    down = torch.clamp(-margin, min=0) + torch.log1p(torch.exp(-margin.abs()))
    loss = ((1 - SMOOTHING) * down + SMOOTHING * (down + margin)).double().mean().float()
    d = (SMOOTHING - torch.sigmoid(-margin)) * (BETA / P)
    d = torch.cat([d, -d])
    if s["starts"] is None:
        dlp = d.expand(s["case"]["length"], -1).reshape(-1)
    else:
        dlp = d[torch.bucketize(torch.arange(len(s["lp"]), device=DEV), s["starts"][1:],
                                right=True)]
    return dict(loss=loss, margin=margin, dlp=dlp)


def _newton_schulz(G):
    """The orthogonalised [k, m, n] by steps of the quintic, in fp32."""
    X = G.float()
    wide = X.shape[1] <= X.shape[2]
    X = X if wide else X.transpose(1, 2).contiguous()
    norm = X.double().square().sum((1, 2), keepdim=True).sqrt()
    X = (X / (norm + NS_EPS)).float()
    for _ in range(NS_STEPS):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = NS[0] * X + torch.bmm(NS[1] * A + NS[2] * torch.bmm(A, A), X)
    return X if wide else X.transpose(1, 2).contiguous()


def _plain_orthogonalize(s):
    return dict(O=_newton_schulz(s["G"]).to(s["G"].dtype))


def _plain_muon(s):
    for p, g, m, master in zip(s["p"], s["g"], s["m"], s["master"]):
        g = g.float()
        m.copy_(MOMENTUM * m + (1 - MOMENTUM) * g)
        O = _newton_schulz((MOMENTUM * m + (1 - MOMENTUM) * g)[None])[0]
        scale = math.sqrt(max(1.0, p.shape[0] / p.shape[1]))
        w = (p.float() if master is None else master) * (1 - LR * DECAY) - (LR * scale) * O
        if master is not None:
            master.copy_(w)
        p.copy_(w)
    return _muon_outputs(s)


PLAIN = {"recurrence": _plain_recurrence, "recurrence_grad": _plain_recurrence_grad,
         "policy": _plain_policy, "preference": _plain_preference,
         "orthogonalize": _plain_orthogonalize, "muon": _plain_muon}


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------

def _products(m, n):
    """Additions and multiplications of the steps: of a symmetric product one half."""
    m, n = min(m, n), max(m, n)
    return NS_STEPS * (m * m * n + m ** 3 + 2 * m * m * n)


def work(case):
    op = case["op"]
    if op.startswith("recurrence"):
        cols = case["T"] * case["batch"]
        n, z = case["H"] * cols, SIZE[case["dtype"]]
        state = 8 * case["H"] * case["batch"] + (cols if case["resets"] else 0)
        if op == "recurrence":
            return dict(bytes=3 * n * z + state, flops=6 * n)
        arrays = 6 if case["form"] == "gate" else 5          # x is not in the linear form's
        return dict(bytes=arrays * n * z + state + 4 * case["H"] * case["batch"], flops=10 * n)
    if op == "policy":
        arrays = 5 + case["reference"] + 2 * case["entropy"]
        return dict(bytes=4 * arrays * case["tokens"] + 12, flops=20 * case["tokens"])
    if op == "preference":
        S = 2 * case["pairs"]
        n = S * case["length"] * (0.5 if case["packed"] else 1)
        return dict(bytes=12 * n + 2 * S + 4 + (8 * (S + 1) if case["packed"] else 0), flops=3 * n)
    if op == "orthogonalize":
        n = case["count"] * case["m"] * case["n"]
        return dict(bytes=2 * SIZE[case["dtype"]] * n,
                    flops=case["count"] * _products(case["m"], case["n"]))
    each = SIZE[case["gdtype"]] + 8 + SIZE[case["dtype"]] + \
        (8 if case["masters"] else SIZE[case["dtype"]])
    shapes = _shapes(case)
    return dict(bytes=each * sum(a * b for a, b in shapes),
                flops=sum(_products(a, b) for a, b in shapes))


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("recurrence"):
        return _exact_recurrence(case, s)
    if op == "policy":
        return _exact_policy(s)
    if op == "preference":
        P = case["pairs"]
        if case["packed"]:
            seq = torch.repeat_interleave(torch.arange(2 * P, device=DEV), s["starts"].diff())
        else:
            seq = torch.arange(2 * P, device=DEV).repeat(case["length"])
        sums = torch.zeros(2 * P, dtype=torch.float64, device=DEV)
        sums.index_add_(0, seq, s["lp"].double() - s["reference"].double())
        sums.requires_grad_()
        margin = BETA * (sums[:P] - sums[P:])
        good, bad = (torch.nn.functional.logsigmoid(v) for v in (margin, -margin))
        loss = -((1 - SMOOTHING) * good + SMOOTHING * bad).mean()
        d, = torch.autograd.grad(loss, sums)
        return dict(loss=loss.detach(), margin=margin.detach(), dlp=d[seq])
    if op == "orthogonalize":
        return dict(O=torch.stack([_exact_newton_schulz(G.double()) for G in s["G"]]))
    out = dict(p=[], m=[], **(dict(master=[]) if case["masters"] else {}))
    for p, g, m, master in zip(s["p"], s["g"], s["m"], s["master"]):
        g = g.double()
        m = torch.lerp(g, m.double(), MOMENTUM)
        O = _exact_newton_schulz(torch.lerp(g, m, MOMENTUM))
        w = (p if master is None else master).double()
        w = w - LR * (DECAY * w + max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * O)
        out["m"].append(m)
        out["p"].append(w)
        if case["masters"]:
            out["master"].append(w)
    return out


def _exact_newton_schulz(G):
    """Through the singular values where that is quick, else by the steps themselves."""
    x = G / (torch.linalg.matrix_norm(G) + NS_EPS)
    if min(x.shape) <= 256:
        U, v, Vh = (t.to(DEV) for t in torch.linalg.svd(x.cpu(), full_matrices=False))
        for _ in range(NS_STEPS):
            v = NS[0] * v + NS[1] * v ** 3 + NS[2] * v ** 5
        return (U * v) @ Vh
    for _ in range(NS_STEPS):
        if x.shape[0] <= x.shape[1]:
            q = x @ x.mT
            x = NS[0] * x + NS[1] * (q @ x) + NS[2] * (q @ (q @ x))
        else:
            q = x.mT @ x
            x = NS[0] * x + NS[1] * (x @ q) + NS[2] * ((x @ q) @ q)
    return x


def _exact_recurrence(case, s):
    H, T, n = case["H"], case["T"], case["batch"]
    at = lambda t: t.double().reshape(H, T, n).transpose(0, 1).contiguous()      # noqa: E731
    z, x = at(s["gate"]), at(s["x"])
    gate = case["form"] == "gate"
    f = torch.special.expit(z) if gate else z
    free = (torch.zeros(T, 1, n, dtype=torch.bool, device=DEV) if s["resets"] is None
            else s["resets"].view(T, 1, n))
    if case["op"] == "recurrence":
        hs, h = torch.empty_like(x), s["h0"].double()
        for t in range(T):                   # step by step
            h = h.masked_fill(free[t], 0.0)
            h = torch.lerp(x[t], h, f[t]) if gate else torch.addcmul(x[t], f[t], h)
            hs[t] = h
        return dict(h=hs.transpose(0, 1).reshape(H, -1), last=h)
    hs, dh = at(s["h"]), at(s["dh"])
    dgate, dx = torch.empty_like(x), torch.empty_like(x)
    g = s["dh_last"].double()
    for t in range(T - 1, -1, -1):
        g = g + dh[t]
        before = (hs[t - 1] if t else s["h0"].double()).masked_fill(free[t], 0.0)
        if gate:
            dgate[t], dx[t] = g * (before - x[t]) * f[t] * (1 - f[t]), g * (1 - f[t])
        else:
            dgate[t], dx[t] = g * before, g
        g = (g * f[t]).masked_fill(free[t], 0.0)
    back = lambda t: t.transpose(0, 1).reshape(H, -1)                            # noqa: E731
    return dict(dgate=back(dgate), dx=back(dx), dh0=g)


def _exact_policy(s):
    lp = s["lp"].double().requires_grad_()
    w, A = s["weight"].double(), s["advantage"].double()
    ratio = (lp - s["old"].double()).exp()
    inside = ((ratio >= 1 - CLIP_LOW) | (A >= 0)) & ((ratio <= 1 + CLIP_HIGH) | (A <= 0))
    bound = torch.where(A >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW).double()
    loss = -(w * torch.where(inside, ratio, bound) * A).sum()
    kl = torch.zeros((), dtype=torch.float64, device=DEV)
    if s["reference"] is not None:
        q = s["reference"].double() - lp
        kl = (w * (q.exp() - 1 - q)).sum()
        loss = loss + KL * kl
    out = {}
    if s["entropy"] is not None:
        loss = loss - ENTROPY * (w * s["entropy"].double()).sum()
        out["dentropy"] = -ENTROPY * w
    d, = torch.autograd.grad(loss, lp)
    return dict(out, loss=loss.detach(), kl=kl.detach(), clipped=(w * ~inside).sum(), dlp=d)
