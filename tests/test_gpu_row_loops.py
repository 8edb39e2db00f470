"""Rotation, appending and reading at sizes where a thread or a block takes more than one
piece of work: heads, units and token groups of a rotation, many tokens a block of a copy."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_token_cache import append, make_rows, rotary, rotated
from token_cache_util import Cache, quantise, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def rotate(torch, r, pos, backward, dtype, x, y, xs, ys):
    sp.sp_rotate(torch.cuda.current_stream(), r, len(pos), pos.cuda(), backward, dtype, x.shape[1], x, *xs, y, *ys)
    torch.cuda.synchronize()


# Heads that a thread takes one after another, units of a head beyond a block's threads, token
# groups of a block (tokens above 2 x 16 blocks x 152 SMs x those a block holds at once).
MANY = [(70, 40, 128, 128), (9, 48, 128, 64), (5, 300, 64, 64), (3, 7, 1024, 1024), (2, 9, 1000, 640), (3, 40, 33, 30),
        (5000, 4, 32, 32), (20000, 6, 64, 32), (21000, 33, 128, 64), (40001, 3, 32, 8), (40001, 2, 6, 2)]


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,dh,rot", MANY)
@pytest.mark.parametrize("place", ["dense", "in place", "odd"])
def test_rotation_of_many_heads_units_and_tokens(torch, dtype, pairs, n, heads, dh, rot, place):
    g = torch.Generator(device="cuda").manual_seed(n + rot)
    pad = {"dense": 0, "in place": 8, "odd": 1}[place]  # (odd: no 16-byte vectors)
    t = torch_type(dtype)
    buf = torch.randn((n, heads + 2, dh + pad), generator=g, device="cuda").to(t)
    x = buf[:, :heads, :dh]
    keep = buf.clone()
    pos = torch.randint(-500, 1 << 20, (n,), dtype=torch.int32, generator=torch.Generator().manual_seed(n))
    r, freq, amp = rotary(torch, dh, rot, pairs, sp.SP_ROPE_LINEAR, factor=3.0)
    strides = (x.stride(0), x.stride(1))
    backward = n & 1
    if place == "in place":
        rotate(torch, r, pos, backward, dtype, x, x, strides, strides)
        got = x.clone()
        buf[:, :heads, :dh] = keep[:, :heads, :dh]
        assert torch.equal(buf, keep)  # nothing between the heads was touched
    else:
        got = torch.full((n, heads, dh), 7.0, device="cuda").to(t)
        rotate(torch, r, pos, backward, dtype, x, got, strides, (heads * dh, dh))
    # every token of short calls, else some hundred of them and the last ones
    some = torch.arange(n) if n < 1000 else torch.cat([torch.randperm(n, generator=torch.Generator().manual_seed(1))[:150],
                                                       torch.arange(n - 20, n)])
    ref, bound = rotated(torch, keep[:, :heads, :dh][some.cuda()], pos[some].tolist(), freq, amp, pairs, backward)
    # (twice the bound for the float64 reference's own rounding of large angles, as for single heads)
    bound = bound * 2 + 2.0 ** -8 * ref.abs() * (dtype == sp.SP_BF16)
    assert bool(((got[some.cuda()].double().cpu() - ref).abs() <= bound).all())
    # and all tokens against calls of single heads over a few hundred tokens each, within twice the
    # rotation's error at elements below 6 and the results' roundings
    one = torch.empty_like(got)
    for h in range(0, heads, max(1, heads // 3)):
        for a in range(0, n, 997):
            b = min(n, a + 997)
            xi = keep[a:b, h:h + 1, :dh]
            sp.sp_rotate(torch.cuda.current_stream(), r, b - a, pos[a:b].cuda(), backward, dtype, 1, xi, *strides,
                         one[a:b, h:h + 1], heads * dh, dh)
        torch.cuda.synchronize()
        a, b = one[:, h].double(), got[:, h].double()
        assert bool(((a - b).abs() <= 2.4e-5 + 2.0 ** -7 * b.abs() * (dtype == sp.SP_BF16)).all())


# ---- append and read: 4864 rows and more, 16 tokens a block -----------------------
SIZES = [(128, 8, 0), (128, 8, 16), (128, 3, 64), (64, 5, 32), (32, 7, 16), (64, 1, 0), (32, 40, 64)]


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("dh,hkv,page", SIZES)
def test_long_prompts_are_appended_and_nothing_else(torch, cdt, dtype, dh, hkv, page):
    lens, count = [0, 15, 700, 3], [1999, 1400, 17, 1301]
    g = torch.Generator().manual_seed(dh + hkv)
    room = [a + b + 2 for a, b in zip(lens, count)]
    cache, want = (Cache(cdt, hkv, dh, room, page, seed=1, junk=3.0) for _ in range(2))
    total = sum(count)
    k, v = ((torch.randn((total, hkv, dh), generator=g) * torch.exp(torch.randn((total, hkv, 1), generator=g) * 3))
            .to(torch_type(dtype)) for _ in range(2))
    rows = make_rows(torch, count, max(count), total, row0=np.cumsum([0] + count)[:-1])
    assert append(torch, cache, lens, rows, dtype, k.cuda(), v.cuda()) == 0
    at = 0
    for s in range(4):
        want.put(s, lens[s], k[at:at + count[s]].float(), v[at:at + count[s]].float())
        at += count[s]
    for a, b in ((cache.k, want.k), (cache.v, want.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if cdt == sp.SP_E4M3:
        for a, b in ((cache.ks, want.ks), (cache.vs, want.vs)):
            assert bool(((a - b).abs() <= 2.0 ** -22 * b.abs()).all())


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("pairs,part", [(False, 1), (True, 1), (False, 2), (True, 2), (False, 3)])
@pytest.mark.parametrize("dh,hkv,page", SIZES)
def test_long_prompts_are_rotated_on_the_way(torch, cdt, dtype, pairs, part, dh, hkv, page):
    lens, n = [5, 700], 2600
    rot = dh // part & ~1
    g = torch.Generator().manual_seed(rot)
    r, freq, amp = rotary(torch, dh, rot, pairs, sp.SP_ROPE_LINEAR, factor=4.0)
    cache = Cache(cdt, hkv, dh, [L + n for L in lens], page)
    k, v = (torch.randn((2 * n, hkv, dh), generator=g).to(torch_type(dtype)) for _ in range(2))
    assert append(torch, cache, lens, make_rows(torch, None, n, 2 * n), dtype, k.cuda(), v.cuda(), r) == 0
    some = torch.cat([torch.arange(0, 40), torch.randperm(n, generator=g)[:120], torch.arange(n - 20, n)])
    for s in range(2):
        ref, bound = rotated(torch, k[s * n + some], [lens[s] + int(j) for j in some], freq, amp, pairs)
        got = cache.values(s, lens[s] + n, "k")[lens[s] + some]
        if cdt == sp.SP_E4M3:  # (the bound of the short prompts' test)
            scale = ref.abs().amax(-1, keepdim=True) / 448
            bound = bound + (ref.abs() * 2.0 ** -4 + 2.0 ** -10 * scale) * (1 + 1e-4) + 1e-5 * ref.abs()
        else:
            bound = bound + 2.0 ** -8 * ref.abs()
        assert bool(((got - ref).abs() <= bound + 1e-12).all())
        want = v[s * n:(s + 1) * n].float()
        if cdt == sp.SP_E4M3:
            assert torch.equal(cache.codes(s, lens[s] + n, "v")[lens[s]:], quantise(want)[0].view(torch.uint8))
        else:
            assert torch.equal(cache.values(s, lens[s] + n, "v")[lens[s]:], want.to(torch.bfloat16).double())


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dh,hkv,page", SIZES)
def test_long_contexts_are_read(torch, cdt, dtype, pad, dh, hkv, page):
    lens, most = [2100, 0, 1300, 37], 1700
    g = torch.Generator().manual_seed(page + dh)
    cache = Cache(cdt, hkv, dh, [x + 1 for x in lens], page)
    for s, n in enumerate(lens):
        cache.put(s, 0, torch.randn((n, hkv, dh), generator=g), torch.randn((n, hkv, dh), generator=g))
    first, count = [400, 0, 3, 0], [most, most, 1290, 40]
    k, v = (torch.full((4, most, hkv * dh + pad), 9.0).to(torch_type(dtype)).cuda() for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = make_rows(torch, count, most, 4 * most, ks=hkv * dh + pad, vs=hkv * dh + pad)
    sp.sp_cache_read(torch.cuda.current_stream(), cache.desc, 4, None, torch.tensor(lens, dtype=torch.int32).cuda(),
                     torch.tensor(first, dtype=torch.int32).cuda(), rows, dtype, k, v, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for s, (f, n) in enumerate(zip(first, count)):
        for out, which in ((k, "k"), (v, "v")):
            x = cache.values(s, lens[s], which)[f:f + n]
            want = torch.zeros((n, hkv, dh), dtype=torch.float64)
            want[:len(x)] = x
            assert torch.equal(out[s, :n, :hkv * dh].cpu().reshape(n, hkv, dh), want.float().to(out.dtype))
            assert bool((out[s, n:] == 9).all()) and bool((out[s, :, hkv * dh:] == 9).all())
