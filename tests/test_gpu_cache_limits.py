"""Lengths that are wrong, and positions at the ends of their range: reported, and nothing
is written or read where it does not belong."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_token_cache import append, make_rows
from test_gpu_tree import tree_call
from token_cache_util import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def bits(t):
    import torch
    return t.view(torch.uint8)


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("short", [0, 10, 4000, 6000])
def test_positions_that_pass_31_bits_are_skipped(torch, cdt, page, short):
    # the largest bound that is accepted, a length `short` below it and more rows than the
    # bound leaves: tokens without a page, tokens past the bound, and none that wrapped
    hkv, dh, most = 2, 128, 2 ** 31 - 1 - 4096
    k = torch.randn((10000, hkv, dh), generator=torch.Generator().manual_seed(1)).cuda()
    cache, want = (Cache(cdt, hkv, dh, [40, 40], page, junk=3.0) for _ in range(2))
    cache.desc.max_seq_len = most
    turns, amplitude = sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, dh)
    turns = torch.from_numpy(turns.view(np.int64)).cuda()
    rot = sp.sp_rotary(dh, dh, 0, amplitude, turns.data_ptr())
    for r in (None, rot):
        status = append(torch, cache, [most - short, 5], make_rows(torch, [5000, 0], 5000, 10000), sp.SP_F32, k, k, r)
        assert status == (sp.SP_DEV_BAD_PAGE if short else 0) | (sp.SP_DEV_BAD_LENGTH if short < 5000 else 0)
        assert torch.equal(bits(cache.k), bits(want.k)) and torch.equal(bits(cache.v), bits(want.v))


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("length", [-1, -3, -2 ** 31])
def test_a_negative_length_appends_nothing(torch, cdt, page, length):
    hkv, dh = 2, 128
    k = torch.randn((12, hkv, dh), generator=torch.Generator().manual_seed(1)).cuda()
    cache, want = (Cache(cdt, hkv, dh, [40, 40, 40], page, junk=3.0) for _ in range(2))
    assert append(torch, cache, [length, 5, length], make_rows(torch, None, 4, 12), sp.SP_F32, k, k) == sp.SP_DEV_BAD_LENGTH
    want.put(1, 5, k[4:8].cpu(), k[4:8].cpu())
    for a, b in ((cache.k, want.k), (cache.v, want.v)):
        assert torch.equal(bits(a), bits(b))
    if cdt == sp.SP_E4M3:
        other = torch.ones_like(cache.ks, dtype=torch.bool)
        other[cache._at(1, np.arange(5, 9))] = False
        assert bool((cache.ks[other] == 1).all()) and bool((cache.vs[other] == 1).all())


@pytest.mark.parametrize("cdt,path", [(sp.SP_BF16, 1), (sp.SP_BF16, 2), (sp.SP_E4M3, 1), (sp.SP_E4M3, 2), (sp.SP_F32, 1)])
@pytest.mark.parametrize("B", [1, 200])
def test_a_length_that_the_page_table_has_no_room_for_is_cut(torch, cdt, path, B):
    # the largest bound that is accepted stands for "none"; a corrupt length ends where the pages do
    hkv, dh, N, most = 2, 128, 5, 2 ** 31 - 1 - 4096
    cache = Cache(cdt, hkv, dh, [64] * B, 16, spare_pages=0)
    g = torch.Generator().manual_seed(3)
    for s in range(B):
        cache.put(s, 0, *(torch.randn((64, hkv, dh), generator=g) for _ in range(2)))
    q, k, v = (torch.randn((B, N, h, dh), generator=g).to(torch.bfloat16).cuda() for h in (4, hkv, hkv))
    dims = sp.sp_tree_dims(4, N, sp.SP_BF16, path, 0, 0.0, 0, 0, 0)
    lens = [64 if s % 3 == 1 else most - s for s in range(B)]
    want, status = tree_call(torch, cache, dims, [64] * B, None, None, q, k, v, max_len=most)
    assert status == 0
    got, status = tree_call(torch, cache, dims, lens, None, None, q, k, v, max_len=most)
    assert status == sp.SP_DEV_BAD_LENGTH and torch.equal(got, want)
