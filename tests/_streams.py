"""What the tests of calls on several streams share."""
import pytest

torch = pytest.importorskip("torch")


class Busy:
    """Some tens of milliseconds of work on the current stream: what is queued behind it is still
    to come while other streams run."""

    def __init__(self):
        self.a = torch.randn(8192, 8192, device="cuda")
        self.out = torch.empty_like(self.a)
        self.queue(1)
        torch.cuda.synchronize()

    def queue(self, times=6):
        for _ in range(times):
            torch.mm(self.a, self.a, out=self.out)


def flat(r):
    """A call's results as a list of tensors (nested tuples and lists opened)."""
    if isinstance(r, (tuple, list)):
        return [t for x in r for t in flat(x)]
    return [] if r is None else [r]


def copies(r):
    return [t.clone() for t in flat(r)]


def same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


def without_native(monkeypatch, d):
    """The calls in Python code: the native module takes none of them."""
    for name in ("spmv", "spmm", "spmv_packed", "spmm_packed", "spmv_i8", "spmm_i8", "encode", "spmm_grad",
                 "token_logprobs", "token_logprobs_grad", "layer_norm", "layer_norm_grad", "adamw_step",
                 "adamw_moments"):
        monkeypatch.setattr(d._native, name, lambda *a: None)
