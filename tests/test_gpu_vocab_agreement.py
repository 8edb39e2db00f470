"""The vocabulary loss's gradients for tokens that are almost sure of their target: g = p - 1 is the difference
of nearly equal numbers, so that the logits of the backward pass have to be the sums whose log sum the forward
pass wrote."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_vocab_loss import HALF, backward, dims_of, forward
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu
CLASSES = 16  # different tokens


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def sure_tokens(torch, n, d, V, dtype, size, seed):
    """n tokens of CLASSES kinds: kind c has the target c with a logit of about `size`, row CLASSES + c with one
    smaller by 6 to 14, and all the others near 0.  The last CLASSES dims are 0 in h and, in the target rows
    alone, a 1 of their own: dimension d - CLASSES + c of dh is g of target c and nothing else."""
    g = torch.Generator().manual_seed(seed)
    t = torch_type(dtype)
    d0 = d - CLASSES
    base = torch.zeros((CLASSES, d))
    base[:, :d0] = torch.randn((CLASSES, d0), generator=g)
    base = base.to(t)
    w = torch.randn((V, d), generator=g) * 0.1 / d ** 0.5
    w[:, d0:] = 0
    sq = (base.double() ** 2).sum(-1)
    gaps = torch.linspace(6.0, 14.0, CLASSES)
    for c in range(CLASSES):
        w[c, :d0] = base[c, :d0].float() * float(size / sq[c])
        w[c, d0 + c] = 1.0
        w[CLASSES + c, :d0] = base[c, :d0].float() * float((size - gaps[c]) / sq[c])
    kind = torch.arange(n) % CLASSES
    return base[kind].cuda(), w.to(t).cuda(), kind.int().cuda()


@pytest.mark.parametrize("dtype,path", [(sp.SP_BF16, 2), (sp.SP_BF16, 1), (sp.SP_F32, 1)])
@pytest.mark.parametrize("n,d,V", [(CLASSES, 1024, 300), (20, 4096, 300), (100, 4104, 700), (300, 4096, 2000),
                                   (20, 8192, 40000), (260, 2568, 20001)])
def test_gradient_of_almost_certain_tokens(torch, dtype, path, n, d, V):
    size = 30.0
    h, w, t = sure_tokens(torch, n, d, V, dtype, size, n + d)
    dims = dims_of(h, w, d, dtype, path)
    _, lse, status = forward(torch, dims, h, w, t)
    assert status == 0
    dh, _, status = backward(torch, dims, h, w, t, lse, None, head=False)
    assert status == 0
    x, y = h.double(), w.double()
    logits = x @ y.T
    row = torch.arange(n, device="cuda")
    rest = torch.exp(logits - logits[row, t.long()][:, None])
    rest[row, t.long()] = 0
    rest = rest.sum(-1)
    want = -rest / (1 + rest)  # p - 1 without a difference
    assert float(want.abs().min()) < 1e-6 and 1e-3 < float(want.abs().max()) < 5e-3
    got = dh[row, d - CLASSES + t.long()].double()
    # the log sum (16 to 32) is rounded to fp32, half a step 2^-20; its logarithm, p's exponential and p - 1 add
    # less than 2^-21 together; what remains is 1 - p, moved by the errors of a difference of two logits
    # (d + 4 steps each) and rounded to the operand's type and to dh's
    step = 2.0 ** -22 if path == 2 else 2.0 ** -24
    off = size * (d + 4) * step
    lim = 2.0 ** -20 + 2.0 ** -21 + want.abs() * (2 * off + HALF[sp.SP_BF16] * (2 if path == 2 else 1))
    err = (got - want).abs() / lim
    print(n, d, V, dtype, path, "worst / limit", float(err.max()), "worst", float((got - want).abs().max()))
    assert bool((err <= 1).all()), (float(err.max()), got[:CLASSES].tolist(), want[:CLASSES].tolist())
