"""The largest batches of the tree attention: the tile tables then leave the rings one or two
slots, and a block walks hundreds of sequences."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_tree import tree_call
from token_cache_util import Cache, mask_tensor, random_parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("B,G,N", [(2048, 4, 3), (2047, 4, 13), (2048, 4, 30), (2048, 4, 40), (2048, 1, 1)])
def test_a_batch_of_two_thousand(torch, cdt, page, B, G, N):
    hkv, dh = 2, 128
    rng = np.random.default_rng(N)
    lens = [int(x) for x in rng.integers(0, 300, B)]
    n_nodes = [int(x) for x in rng.integers(0, N + 1, B)]
    cache = Cache(cdt, hkv, dh, [max(x, 1) for x in lens], page, junk=0.0)
    g = torch.Generator(device="cuda").manual_seed(N)
    for pool in (cache.k, cache.v):
        pool.copy_(torch.randn(pool.shape, generator=g, device="cuda").mul_(1 if cdt == sp.SP_BF16 else 60).to(pool.dtype))
    if cdt == sp.SP_E4M3:
        for sc in (cache.ks, cache.vs):
            sc.copy_(torch.rand(sc.shape, generator=g, device="cuda") / 40)
    q, k, v = (torch.randn((B, N, h, dh), generator=g, device="cuda").to(torch.bfloat16) for h in (G * hkv, hkv, hkv))
    trees = [sp.sp_tree_masks(random_parents(rng, N))[0] for _ in range(64)]
    masks = mask_tensor(torch, np.stack([trees[b % 64] for b in range(B)]))
    dims = sp.sp_tree_dims(G * hkv, N, sp.SP_BF16, 2, 0, 0.0, 0, 0, 0)
    got, status = tree_call(torch, cache, dims, lens, masks, n_nodes, q, k, v)
    assert status == 0
    again, _ = tree_call(torch, cache, dims, lens, masks, n_nodes, q, k, v)
    assert torch.equal(got, again)
    dims.path = 1
    ref, _ = tree_call(torch, cache, dims, lens, masks, n_nodes, q, k, v)
    # two bf16 roundings of the result and weights of 8 bits, 2^-8 each: of every sequence's 2-norm
    off, size = ((x.double().flatten(1)).norm(dim=1) for x in (got.double() - ref.double(), ref))
    assert bool((off <= 3 * 2.0 ** -8 * size).all())
    dead = torch.arange(N)[None] >= torch.tensor(n_nodes)[:, None]
    assert bool((got[dead] == 0).all())


def test_a_larger_batch_runs_on_cuda_cores(torch):
    hkv, dh, N, B = 2, 128, 2, 2049
    cache = Cache(sp.SP_BF16, hkv, dh, [3] * B, 16, junk=0.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    for pool in (cache.k, cache.v):
        pool.copy_(torch.randn(pool.shape, generator=g, device="cuda"))
    q, k, v = (torch.randn((B, N, hkv, dh), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    outs = [tree_call(torch, cache, sp.sp_tree_dims(hkv, N, sp.SP_BF16, path, 0, 0.0, 0, 0, 0), [3] * B, None, None, q, k, v)[0]
            for path in (0, 1)]
    assert torch.equal(*outs)
    with pytest.raises(sp.SpError) as e:
        sp.sp_attend_tree(None, sp.sp_tree_dims(hkv, N, sp.SP_BF16, 2, 0, 0.0, 0, 0, 0), cache.desc, B, None, q, None, None, q, k, v,
                          q, q, 1 << 40)
    assert e.value.status == sp.SP_ERR_UNSUPPORTED
