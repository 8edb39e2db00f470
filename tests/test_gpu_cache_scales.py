"""The 8-bit cache's scales are the documented products, bit for bit."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_token_cache import append, make_rows
from token_cache_util import Cache, quantise, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("dh,hkv", [(128, 2), (64, 3), (32, 5)])
def test_scales_are_the_largest_element_times_a_constant(torch, dtype, page, dh, hkv):
    n = 700
    g = torch.Generator().manual_seed(dh + page)
    k, v = ((torch.randn((n, hkv, dh), generator=g) * torch.exp(torch.randn((n, hkv, 1), generator=g) * 8))
            .to(torch_type(dtype)) for _ in range(2))
    k[3], v[5], k[7] = 0.0, 2.0 ** -70, 3e38
    cache = Cache(sp.SP_E4M3, hkv, dh, [n], page)
    assert append(torch, cache, [0], make_rows(torch, None, n, n), dtype, k.cuda(), v.cuda()) == 0
    for which, x in (("k", k), ("v", v)):
        amax = np.maximum(x.float().abs().amax(-1).numpy(), np.float32(2.0 ** -60))
        assert torch.equal(cache.scales(0, n, which), torch.from_numpy(amax * (np.float32(1.0) / np.float32(448.0))))
        assert torch.equal(cache.codes(0, n, which), quantise(x.float())[0].view(torch.uint8))
