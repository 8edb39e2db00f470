"""Vocabulary loss gradients on tensor cores where g does not fit its share of the workspace: the vocabulary is
taken in pieces, the last one shorter.  The workspace's size says that it was (g of the whole vocabulary
would not fit it)."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_vocab_loss import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def in_pieces(n, d, V):
    dims = sp.sp_vocab_dims(n, V, d, sp.SP_BF16, 2, 0, 0)
    return sp.sp_vocab_loss_backward_workspace_bytes(dims) < -(-n // 256) * 256 * V * 2


@pytest.mark.parametrize("head", [True, False])
@pytest.mark.parametrize("n,d,V,skip", [
    (8003, 16, 33500, 0.1),       # two pieces, dh in two parts
    (8003, 264, 33500, 0.0),      # dh's tiles in one part that the second piece adds to
    (200, 8, 1100000, 0.1),       # one tile of tokens, whose W is asked for in front of the count; sixteen parts of dh
    (32768, 16, 24000, 0.99),     # three pieces for few kept tokens: dh in sixteen parts, the last of which gets nothing
                                  # from the last piece
    (32768, 16, 24000, 1.0),      # no token has a target
])
def test_a_vocabulary_in_pieces_on_tensor_cores(torch, n, d, V, skip, head):
    assert in_pieces(n, d, V)
    check(torch, n, d, V, sp.SP_BF16, 2, skip=skip, head=head, seed=n + V)


def test_targets_on_both_sides_of_a_cut(torch):
    # every target lies at an edge of a piece (two of 66 tiles of 256 rows) or of a tile beside it
    from test_gpu_vocab_loss import backward, dims_of, forward, inputs
    n, d, V, cut = 8003, 16, 33500, 66 * 256
    assert in_pieces(n, d, V)
    h, w, t, gl = inputs(torch, n, d, V, sp.SP_BF16, 7)
    edges = torch.tensor([0, cut - 257, cut - 256, cut - 1, cut, cut + 1, cut + 255, cut + 256, V - 1], dtype=torch.int32)
    t = edges[torch.arange(n) % len(edges)].cuda()
    dims = dims_of(h, w, d, sp.SP_BF16, 2)
    loss, lse, status = forward(torch, dims, h, w, t)
    dh, dw, status2 = backward(torch, dims, h, w, t, lse, gl)
    assert status == 0 and status2 == 0
    x, y, up = h.double(), w.double(), gl.double()[:, None]
    p = torch.softmax(x @ y.T, -1)
    p[torch.arange(n, device="cuda"), t.long()] -= 1
    p *= up
    # g to bf16, sums in fp32 (2^-22 a step), the result to bf16; logits of 20 products of sum |h w| below 30
    for got, want, size, k in ((dh, p @ y, p.abs() @ y.abs(), V), (dw, p.T @ x, p.T.abs() @ x.abs(), n)):
        lim = size * (2.0 ** -8 + 30 * 20 * 2.0 ** -21 + min((k + 8) * 2.0 ** -22, 2.0 ** -9)) + want.abs() * 2.0 ** -8 + 1e-38
        assert bool(((got.double() - want).abs() <= lim).all()), float(((got.double() - want).abs() / lim).max())
