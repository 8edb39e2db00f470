"""Rotation of heads of an odd number of dims."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_token_cache import rotary, rotated
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,dh,rot", [(3, 2, 3, 2), (40, 3, 5, 4), (7, 300, 33, 16), (2, 5, 129, 128), (9, 1, 1023, 2),
                                            (50000, 3, 9, 8)])
@pytest.mark.parametrize("backward", [0, 1])
def test_every_dim_arrives(torch, dtype, pairs, n, heads, dh, rot, backward):
    g = torch.Generator().manual_seed(dh)
    x = torch.randn((n, heads, dh), generator=g).to(torch_type(dtype))
    pos = torch.randint(0, 10000, (n,), generator=g, dtype=torch.int32)
    r, freq, amp = rotary(torch, dh, rot, pairs)
    flat = torch.full((n * heads * dh + 8,), 7.0).to(x.dtype).cuda()
    y = flat[:-8].view(n, heads, dh)
    sp.sp_rotate(torch.cuda.current_stream(), r, n, pos.cuda(), backward, dtype, heads, x.cuda(), heads * dh, dh, y, heads * dh, dh)
    torch.cuda.synchronize()
    ref, bound = rotated(torch, x, pos.tolist(), freq, amp, pairs, backward)
    bound = bound + 2.0 ** -8 * ref.abs() * (dtype == sp.SP_BF16)
    assert bool(((y.double().cpu() - ref).abs() <= bound).all())
    assert torch.equal(y[..., rot:].cpu(), x[..., rot:]) and bool((flat[-8:] == 7).all())
