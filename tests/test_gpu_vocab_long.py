"""Vocabulary loss gradients that are sums over many tokens or a large vocabulary: equal terms are rounded the
same way at every step, so that the errors of one long sum add up instead of cancelling."""
import math

import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_vocab_loss import HALF, backward, dims_of, forward
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def equal_rows(torch, n, d, V, dtype):
    """n equal tokens, V equal rows but for row 0, everyone's target, which is their opposite."""
    t = torch_type(dtype)
    g = torch.Generator().manual_seed(V + d)
    h = torch.full((1, d), 0.37)
    h[:, ::2] = -0.61
    w = torch.rand((1, d), generator=g) * 0.5 + 0.3
    h, w = h.to(t).cuda().expand(n, d).contiguous(), w.to(t).cuda().expand(V, d).contiguous().clone()
    w[0] *= -1
    return h, w, torch.zeros(n, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("n,d,V,head", [(65536, 16, 70, True), (500000, 24, 33, True), (4000000, 16, 70, True),
                                        (3, 16, 131072, False), (3, 40, 1 << 20, False), (3, 16, 1 << 24, False),
                                        (70, 40, 200000, True)])
def test_long_sums_on_cuda_cores(torch, dtype, n, d, V, head):
    h, w, t = equal_rows(torch, n, d, V, dtype)
    dims = dims_of(h, w, d, dtype, 1)
    _, lse, _ = forward(torch, dims, h, w, t)
    dh, dw, status = backward(torch, dims, h, w, t, lse, None, head)
    assert status == 0
    x, y = h[0].double(), w[:2].double()
    l0, l1 = float(y[0] @ x), float(y[1] @ x)
    top = max(l0, l1)
    want = top + math.log((V - 1) * math.exp(l1 - top) + math.exp(l0 - top))
    rest = (V - 1) * math.exp(l1 - want)            # 1 - p of the target
    p1 = math.exp(l1 - want)
    # a weight: its logit d + 4 steps, the log sum as in test_gpu_vocab_loss; the target's is a difference from 1
    off = float(x.abs() @ y[1].abs()) * (d + 4) * STEP
    rel = 2 * off + 2.0 ** -16 + abs(want) * 2.0 ** -20
    g0 = rest * rel + 2.0 ** -22
    # a sum: 512 products in one number and what joins such numbers, groups of threads, splits (at most 16) or pieces
    # of the vocabulary (48 at most here) without more; then the result's type
    run = (512 + 64) * STEP
    size = rest * y[0].abs() + rest * y[1].abs()
    exact = -rest * y[0] + rest * y[1]
    lim = y[0].abs() * g0 + rest * y[1].abs() * rel + size * run + exact.abs() * HALF[dtype]
    err = float(((dh.double() - exact).abs() / lim).max())
    print("dh", n, d, V, dtype, err, float(((dh.double() - exact).abs() / size).max()))
    assert err <= 1
    if head:
        for row, g, ge in ((0, -rest, g0), (V - 1, p1, p1 * rel)):
            exact = n * g * x
            lim = n * x.abs() * ge + exact.abs() * (run + HALF[dtype])
            err = float(((dw[row].double() - exact).abs() / lim).max())
            print("dw", row, n, d, V, dtype, err, float(((dw[row].double() - exact) / exact).abs().max()))
            assert err <= 1


@pytest.mark.parametrize("n", [40000, 1000003, 4000000])
@pytest.mark.parametrize("d", [16, 264])
def test_head_gradient_of_many_tokens_on_tensor_cores(torch, n, d):
    # two equal rows: every weight is a half, and its gradient a half in bf16, too
    g = torch.Generator().manual_seed(d)
    h = (torch.rand((1, d), generator=g) + 0.3).to(torch.bfloat16).cuda().expand(n, d).contiguous()
    w = torch.full((2, d), 0.25, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(n, dtype=torch.int32, device="cuda")
    t[::3] = -1
    kept = int((t == 0).sum())
    dims = dims_of(h, w, d, sp.SP_BF16, 2)
    _, lse, _ = forward(torch, dims, h, w, t)
    _, dw, status = backward(torch, dims, h, w, t, lse, None)
    assert status == 0
    # an accumulator's sum is cut at its 24 bits 1024 times at most (16384 tokens, 16 a step), each by less than one
    # part in 2^23 of it; accumulators are added in fp32 (244 at most); then bf16
    for row, sign in ((0, -0.5), (1, 0.5)):
        exact = sign * kept * h[0].double()
        err = ((dw[row].double() - exact) / exact).abs().max()
        print("dw", n, d, row, float(err))
        assert float(err) <= 2.0 ** -8 + 1024 * 2.0 ** -23 + 244 * STEP
