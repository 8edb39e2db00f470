"""Offsets past 32 bits: rotations of more than 2^31 elements, caches of more than 2^32."""
import types

import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_token_cache import append, make_rows, rotary, rotated
from token_cache_util import quantise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_of_more_than_2_31_elements(torch, pairs):
    n, heads, dh, rot = 141000, 120, 128, 64
    x = torch.empty((n, heads, dh), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    assert x.numel() > 2 ** 31
    some = torch.tensor([0, 1, n // 2, n - 20, n - 2, n - 1])
    keep = x[some.cuda()].clone()
    pos = torch.arange(n, dtype=torch.int32) * 7
    r, freq, amp = rotary(torch, dh, rot, pairs)
    sp.sp_rotate(torch.cuda.current_stream(), r, n, pos.cuda(), 0, sp.SP_BF16, heads, x, heads * dh, dh, x, heads * dh, dh)
    torch.cuda.synchronize()
    ref, bound = rotated(torch, keep, pos[some].tolist(), freq, amp, pairs)
    assert bool(((x[some.cuda()].double().cpu() - ref).abs() <= bound * 2 + 2.0 ** -8 * ref.abs()).all())


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("paged", [True, False])
def test_appending_and_reading_past_2_32_elements(torch, cdt, paged):
    # one sequence's tokens at the far end of the pool (paged), or past 2^22 tokens of 1024 elements
    hkv, dh, P, n = 8, 128, 64, 150
    first = 2 ** 32 // (hkv * dh) + 37
    room = -(-(first + n) // P) * P
    shape = (room // P, hkv, P, dh) if paged else (room, hkv, dh)
    kind = torch.uint8 if cdt == sp.SP_E4M3 else torch.bfloat16
    k_pool, v_pool = (torch.zeros(shape, dtype=kind, device="cuda") for _ in range(2))
    scales = [torch.zeros(shape[:-1], device="cuda") for _ in range(2)]
    assert k_pool.numel() > 2 ** 32
    table = torch.arange(room // P, dtype=torch.int32, device="cuda")[None].contiguous()
    ptrs = [torch.tensor([t.data_ptr()], dtype=torch.int64, device="cuda") for t in (k_pool, v_pool, *scales)]
    if paged:
        kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, k_pool.data_ptr(), v_pool.data_ptr(), table.data_ptr(), P, room // P,
                            room // P, 1)
        sc = [t.data_ptr() for t in scales]
    else:
        kv = sp.sp_kv_cache(sp.SP_KV_CONTIGUOUS, ptrs[0].data_ptr(), ptrs[1].data_ptr(), None, None, None, 0, 0, 0, 1)
        sc = [t.data_ptr() for t in ptrs[2:]]
    desc = sp.sp_token_cache(kv, cdt, hkv, dh, room, *(sc if cdt == sp.SP_E4M3 else (None, None)))
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((n, hkv, dh), generator=g).to(torch.bfloat16) for _ in range(2))

    cache = types.SimpleNamespace(desc=desc)
    assert append(torch, cache, [first], make_rows(torch, None, n, n), sp.SP_BF16, k.cuda(), v.cuda()) == 0
    outs = [torch.empty((n, hkv, dh), device="cuda") for _ in range(2)]
    at = torch.tensor([first], dtype=torch.int32, device="cuda")
    rows = make_rows(torch, None, n, n)
    sp.sp_cache_read(torch.cuda.current_stream(), desc, 1, None, at + n, at, rows, sp.SP_F32, *outs)
    torch.cuda.synchronize()
    for out, x in zip(outs, (k, v)):
        want = x.float()
        if cdt == sp.SP_E4M3:
            codes, scale = quantise(want)
            want = codes.float() * scale[..., None]
        assert bool(((out.cpu() - want).abs() <= 2.0 ** -22 * want.abs()).all())
    # nothing was written in front of them
    for pool in (k_pool, v_pool):
        flat = pool.view(torch.uint8).view(shape[0], -1)
        start = first // P if paged else first
        for a in range(0, start, 1 << 16):
            assert not bool(flat[a:min(a + (1 << 16), start)].any())
