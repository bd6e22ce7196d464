"""Batches of matrices whose rows lie in turn, as results of the orthogonalised update."""
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import TYPES  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("k,m,n", [(3, 70, 130), (2, 1, 9), (5, 40, 1), (4, 33, 64)])
def test_rows_in_turn(darb, dtype, k, m, n):
    g = torch.randn(k, m, n, device="cuda").to(TYPES[dtype])
    want = darb.orthogonalize(g)
    inside = torch.full((m, k + 2, n + 3), 9.0, device="cuda", dtype=TYPES[dtype])
    view = inside[:, 1:k + 1, 2:n + 2].transpose(0, 1)      # [k, m, n], a row of every matrix in turn
    view.copy_(g)
    assert torch.equal(darb.orthogonalize(view), want)
    assert darb.orthogonalize(view, out=view) is view and torch.equal(view, want)
    assert (inside[:, 0] == 9).all() and (inside[:, k + 1] == 9).all()
    assert (inside[:, :, :2] == 9).all() and (inside[:, :, n + 2:] == 9).all()
    # transposed matrices in turn
    turned = torch.full((n, k, m), 9.0, device="cuda", dtype=TYPES[dtype]).permute(1, 2, 0)
    turned.copy_(g)
    assert torch.equal(darb.orthogonalize(turned, out=turned), darb.orthogonalize(g.mT.contiguous().mT))


def test_overlapping_results_are_refused(darb):
    g = torch.randn(3, 8, 16, device="cuda")
    room = torch.zeros(3 * 8 * 16, device="cuda")
    for strides in ((0, 16, 1), (8, 16, 1), (16, 40, 1), (15, 48, 1), (127, 16, 1), (8, 48, 1)):
        with pytest.raises(ValueError, match="overlap"):
            darb.orthogonalize(g, out=room.as_strided((3, 8, 16), strides))
    assert not room.any()
