"""The evaluation and retraining calls together: one step of the example's layer against the same
mathematics in 64 bits, and a short retraining that brings perplexity down."""
import importlib.util
import os

import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(darb):  # noqa: F811
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "retrain_output_layer.py")
    spec = importlib.util.spec_from_file_location("retrain_output_layer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def f64_step(W, mask, gamma, beta, h, words):
    """(mean log probability, d masked W, d gamma, d beta) of minus that mean, on the CPU."""
    W, gamma, beta = (t.detach().clone().requires_grad_() for t in (W, gamma, beta))
    x = torch.nn.functional.layer_norm(h.t(), (h.shape[0],), gamma, beta, 1e-5).t()
    logp = torch.log_softmax(W @ x, 0)
    mean = logp.gather(0, words[None, :]).mean()
    (-mean).backward()
    return mean.item(), W.grad[mask], gamma.grad, beta.grad


@pytest.mark.parametrize("values", ["f32", "f16"])
@pytest.mark.parametrize("V,H,B", [(257, 96, 50), (90, 133, 1), (1000, 300, 129)])
def test_step_gradients(darb, example, V, H, B, values):  # noqa: F811
    say(f"retraining step: V {V} H {H} B {B} {values}")
    rng = np.random.default_rng(V)
    W = torch.from_numpy(rng.standard_normal((V, H)).astype(np.float32)).cuda() * (3.0 / H ** 0.5)
    h, words, _ = example.make_data(W, B, 1)
    plan, v, o = example.prune(W, 0.1, 4, 16, example.TYPES[values])
    layer = example.OutputLayer(plan, v, o, H)
    layer.weight.copy_(torch.from_numpy(1 + 0.2 * rng.standard_normal(H)))
    layer.bias.copy_(torch.from_numpy(0.2 * rng.standard_normal(H)))
    logprob, (dv, dw, db) = layer.gradients(h, words)
    # where each retained value stands: decode an index in its place (exact in fp32)
    ids = plan.decode(torch.arange(1, plan.nnz + 1, device="cuda", dtype=torch.float32), o)
    dense = plan.decode(layer.values.float(), o)
    torch.cuda.synchronize()
    mask = ids.cpu() > 0
    order = ids.cpu()[mask].long() - 1
    want = f64_step(dense.cpu().double(), mask, layer.weight.cpu().double(),
                    layer.bias.cpu().double(), h.cpu().double(), words.cpu())
    # Relative to the largest gradient: log probabilities of size L carry about 1e-6 L of fp32
    # error (sums of H and V terms, an exponential), and the later sums average over it.
    size = 1e-5 * max(1.0, abs(want[0]))
    assert abs(logprob.item() - want[0]) <= size * 2
    got = dv.cpu().double()[order]
    for g, w in ((got, want[1]), (dw.cpu().double(), want[2]), (db.cpu().double(), want[3])):
        assert g.shape == w.shape
        assert (g - w).abs().max() <= 4 * size * w.abs().max() + 1e-12


@pytest.mark.parametrize("values,bits", [("f32", 32), ("f16", 8)])
def test_retraining_lowers_perplexity(darb, example, values, bits):  # noqa: F811
    say(f"retraining: {values} values, {bits}-bit states")
    args = ["--words", "500", "--hidden", "128", "--keep", "0.1", "--batch", "256", "--batches", "40",
            "--steps", "80", "--values", values, "--state-bits", str(bits)]
    dense, pruned, after = example.main(args)
    assert dense < after < pruned
