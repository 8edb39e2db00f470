"""Gradients of a few tokens against a vocabulary, thousands of times at different distances from the work in front:
a wait that depends on which CTA of a pair comes first shows in some of them (as SP_DEV_TIMEOUT)."""
import random

import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_vocab_loss import backward, dims_of, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


# k-blocks of 64: 1, 4, 9 (more than the six stages); 128 tokens and fewer copy the first CTA's rows alone
@pytest.mark.parametrize("n,d,V", [(9, 16, 40), (1, 520, 2049), (4, 256, 300), (128, 64, 700), (129, 64, 700)])
@pytest.mark.parametrize("side", [False, True])
def test_few_tokens_again_and_again(torch, n, d, V, side):
    h, w, t, gl = inputs(torch, n, d, V, sp.SP_BF16, n + V, skip=0.1 if n > 1 else 0.0)
    dims = dims_of(h, w, d, sp.SP_BF16, 2)
    _, lse, _ = forward(torch, dims, h, w, t)
    want = backward(torch, dims, h, w, t, lse, gl)
    assert want[2] == 0
    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    size = sp.sp_vocab_loss_backward_workspace_bytes(dims)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    junk = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rng = random.Random(n)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for i in range(400):
            if rng.random() < 0.3:
                junk[:rng.randrange(1, 1 << 24)].zero_()
            if rng.random() < 0.5:
                torch.cuda.synchronize()
            sp.sp_vocab_loss_backward(stream, dims, h, w, t, lse, gl, dh, dw, ws, size, status)
            if i % 100 == 99:
                torch.cuda.synchronize()
                assert int(status) == 0, i
    torch.cuda.synchronize()
    assert torch.equal(dh, want[0]) and torch.equal(dw, want[1])
