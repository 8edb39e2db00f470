"""Rotary positions, appending to a token cache and reading it back, against float64."""
import math

import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from token_cache_util import Cache, quantise, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def rotary(torch, dh, rot, pairs, kind=sp.SP_ROPE_PLAIN, **kw):
    turns, amp = sp.sp_rotary_plan(kind, rot, **kw)
    t = torch.from_numpy(turns.view(np.int64)).cuda()
    r = sp.sp_rotary(dh, rot, int(pairs), amp, t.data_ptr())
    r.keep = t
    return r, np.array([int(x) / 2.0 ** 64 for x in turns]), amp


def rotated(torch, x, pos, freq, amp, pairs, backward=False):
    """Float64 rotation of x [n][heads][dh]; freq in turns a position.  Also the bound of
    the fp32 error: angles to 2 pi 2^-32 + pi 2^-24, sincospi to 2 ulp, three roundings
    of the products, the amplitude's two: below 1e-6 a (|u| + |v|)."""
    x = x.double().cpu()
    r = len(freq)
    frac = torch.from_numpy(np.array([[math.fmod(float(p) * f, 1.0) for f in freq] for p in pos]))
    c, s = torch.cos(2 * math.pi * frac)[:, None] * amp, torch.sin(2 * math.pi * frac)[:, None] * amp
    s = -s if backward else s
    u, v = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if pairs else (x[..., :r], x[..., r:2 * r])
    y, e = x.clone(), torch.zeros_like(x)
    p, q, b = u * c - v * s, v * c + u * s, 1e-6 * amp * (u.abs() + v.abs())
    if pairs:
        y[..., 0:2 * r:2], y[..., 1:2 * r:2] = p, q
        e[..., 0:2 * r:2], e[..., 1:2 * r:2] = b, b
    else:
        y[..., :r], y[..., r:2 * r] = p, q
        e[..., :r], e[..., r:2 * r] = b, b
    return y, e


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,dh,rot", [(1, 1, 128, 128), (7, 3, 128, 64), (300, 5, 64, 64), (33, 2, 32, 30),
                                            (2500, 4, 96, 32), (5, 3, 70, 70), (9, 2, 128, 2)])
@pytest.mark.parametrize("backward", [0, 1])
def test_rotation(torch, dtype, pairs, n, heads, dh, rot, backward):
    g = torch.Generator().manual_seed(n * 7 + rot)
    x = torch.randn((n, heads, dh), generator=g).to(torch_type(dtype))
    pos = torch.randint(-5000, 1 << 20, (n,), generator=g, dtype=torch.int32)
    pos[0] = 2 ** 31 - 1 if n > 1 else 0
    # (theta^(-2i/rot) below 2^-31 rounds in the double's last place: exact enough up to here)
    r, freq, amp = rotary(torch, dh, rot, pairs, sp.SP_ROPE_DIMS if rot > 2 else sp.SP_ROPE_PLAIN, factor=4.0,
                          trained_len=4096.0)
    xd, y = x.cuda(), torch.full((n, heads, dh), 7.0).to(x.dtype).cuda()
    sp.sp_rotate(torch.cuda.current_stream(), r, n, pos.cuda(), backward, dtype, heads, xd, heads * dh, dh, y, heads * dh, dh)
    torch.cuda.synchronize()
    ref, bound = rotated(torch, x, pos.tolist(), freq, amp, pairs, backward)
    # (a position near 2^31 times a frequency rounded to 2^-64 turn, in the reference's
    # float64 product: 2^31 2^-53 turns)
    bound = bound * 2 + 2.0 ** -8 * ref.abs() * (dtype == sp.SP_BF16)
    assert bool(((y.double().cpu() - ref).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 3), (0, 8), (2, 5)])
def test_strides_alignment_and_in_place(torch, dtype, offset, pad):
    n, heads, dh, rot = 37, 3, 64, 48
    t = torch_type(dtype)
    th, tt = dh + pad, heads * (dh + pad) + 2 * pad
    flat = torch.randn(offset + n * tt + 16, generator=torch.Generator().manual_seed(3)).to(t).cuda()
    before = flat.clone()
    view = flat[offset:].as_strided((n, heads, dh), (tt, th, 1), flat.storage_offset() + offset)
    pos = torch.arange(n, dtype=torch.int32).cuda() * 11
    r, freq, amp = rotary(torch, dh, rot, False)
    dense = torch.empty((n, heads, dh), dtype=t, device="cuda")
    ptr = view.data_ptr()
    sp.sp_rotate(torch.cuda.current_stream(), r, n, pos, 0, dtype, heads, ptr, tt, th, dense, heads * dh, dh)
    sp.sp_rotate(torch.cuda.current_stream(), r, n, pos, 0, dtype, heads, ptr, tt, th, ptr, tt, th)
    torch.cuda.synchronize()
    assert torch.equal(view, dense)
    ref, bound = rotated(torch, before.as_strided((n, heads, dh), (tt, th, 1), offset), pos.tolist(), freq, amp, False)
    assert bool(((dense.double().cpu() - ref).abs() <= bound + 2.0 ** -8 * ref.abs() * (dtype == sp.SP_BF16)).all())
    # nothing between the heads was touched
    flat.as_strided((n, heads, dh), (tt, th, 1), offset).copy_(before.as_strided((n, heads, dh), (tt, th, 1), offset))
    assert torch.equal(flat, before)


@pytest.mark.parametrize("pairs", [False, True])
def test_the_backward_pass_is_the_adjoint_and_matches_differences(torch, pairs):
    n, heads, dh, rot = 6, 2, 32, 24
    g = torch.Generator().manual_seed(5)
    x, w = (torch.randn((n, heads, dh), generator=g).cuda() for _ in range(2))
    pos = torch.randint(0, 9000, (n,), generator=g, dtype=torch.int32).cuda()
    r, _, _ = rotary(torch, dh, rot, pairs, sp.SP_ROPE_DIMS, factor=8.0, trained_len=1024.0)

    def call(t, backward):
        y = torch.empty_like(t)
        sp.sp_rotate(torch.cuda.current_stream(), r, n, pos, backward, sp.SP_F32, heads, t, heads * dh, dh, y, heads * dh, dh)
        torch.cuda.synchronize()
        return y.double()
    fwd, bwd = call(x, 0), call(w, 1)
    # <w, R x> = <R^T w, x>: each side sums 384 products of fp32 results off by < 4e-6
    assert abs(float((w.double() * fwd).sum() - (bwd * x.double()).sum())) < 384 * 4e-6 * 9
    # the loss <w, R x> is linear: a central difference is exact up to fp32 rounding of
    # its two outputs (|R x| < 8: 2^-20 each) over the step
    for at in [(0, 0, 0), (2, 1, 11), (3, 0, 23), (5, 1, 30)]:
        step = torch.zeros_like(x)
        step[at] = 0.5
        slope = float((w.double() * (call(x + step, 0) - call(x - step, 0))).sum())
        assert abs(slope - float(bwd[at])) < dh * 2.0 ** -19 * 4 + 1e-5


def test_no_tokens_is_a_no_op(torch):
    r, _, _ = rotary(torch, 64, 64, False)
    sp.sp_rotate(torch.cuda.current_stream(), r, 0, None, 0, sp.SP_BF16, 2, None, 128, 64, None, 128, 64)


# ---- append and read --------------------------------------------------------
LAYOUTS = [0, 16, 32, 64]


def append(torch, cache, lens, rows, dtype, k, v, rot=None, ids=None, batch=None):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sp.sp_cache_append(torch.cuda.current_stream(), cache.desc, rot, batch or len(lens), ids,
                       torch.tensor(lens, dtype=torch.int32).cuda(), rows, dtype, k, v, status)
    torch.cuda.synchronize()
    return int(status.item())


def make_rows(torch, count, max_rows, total, row0=None, take=None, ks=0, vs=0):
    keep = [None if x is None else torch.tensor(x, dtype=torch.int32).cuda() for x in (row0, count, take)]
    r = sp.sp_token_rows(*[None if x is None else x.data_ptr() for x in keep], max_rows, total, ks, vs)
    r.keep = keep
    return r


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("page", LAYOUTS)
@pytest.mark.parametrize("dh,hkv", [(128, 2), (64, 3), (32, 1)])
def test_append_writes_its_tokens_and_nothing_else(torch, cdt, dtype, page, dh, hkv):
    lens, count = [0, 15, 16, 40, 63], [3, 1, 0, 29, 2]
    g = torch.Generator().manual_seed(dh + page)
    cache = Cache(cdt, hkv, dh, [a + b + 2 for a, b in zip(lens, count)], page, seed=1, junk=3.0)
    total = sum(count)
    k, v = ((torch.randn((total, hkv, dh), generator=g) * torch.exp(torch.randn((total, hkv, 1), generator=g) * 3))
            .to(torch_type(dtype)) for _ in range(2))
    k[1] = 0.0
    before = [cache.codes(s, lens[s], w) for s in range(5) for w in "kv"]
    pools = [t.clone() for t in (cache.k, cache.v)]
    rows = make_rows(torch, count, max(count), total, row0=np.cumsum([0] + count)[:-1])
    assert append(torch, cache, lens, rows, dtype, k.cuda(), v.cuda()) == 0
    at = 0
    want = Cache(cdt, hkv, dh, cache.room, page, seed=1, junk=3.0)
    for s in range(5):
        want.put(s, lens[s], k[at:at + count[s]].float(), v[at:at + count[s]].float())
        at += count[s]
    for a, b in ((cache.k, want.k), (cache.v, want.v)):  # every bit of the pools
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if cdt == sp.SP_E4M3:  # one division, rounded once or twice
        for a, b in ((cache.ks, want.ks), (cache.vs, want.vs)):
            assert bool(((a - b).abs() <= 2.0 ** -22 * b.abs()).all())
    assert before and pools


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16])
@pytest.mark.parametrize("pairs,rot", [(False, 128), (True, 64), (False, 36), (True, 6), (False, 4)])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
def test_append_rotates_keys_at_their_positions(torch, cdt, pairs, rot, dtype):
    lens, n, hkv, dh = [5, 0, 700], 21, 2, 128
    g = torch.Generator().manual_seed(rot)
    r, freq, amp = rotary(torch, dh, rot, pairs, sp.SP_ROPE_LINEAR, factor=4.0)
    cache = Cache(cdt, hkv, dh, [L + n for L in lens], 16)
    k, v = (torch.randn((3 * n, hkv, dh), generator=g).to(torch_type(dtype)) for _ in range(2))
    assert append(torch, cache, lens, make_rows(torch, None, n, 3 * n), dtype, k.cuda(), v.cuda(), r) == 0
    for s in range(3):
        ref, bound = rotated(torch, k[s * n:(s + 1) * n], range(lens[s], lens[s] + n), freq, amp, pairs)
        got = cache.values(s, lens[s] + n, "k")[lens[s]:]
        if cdt == sp.SP_E4M3:
            # half a step of 3 mantissa bits, or of the 2^-9 below the smallest normal
            # value, scale included, and the step the rotation's error can move it to
            scale = (ref.abs().amax(-1, keepdim=True) / 448).clamp_min(0)
            bound = bound + (ref.abs() * 2.0 ** -4 + 2.0 ** -10 * scale) * (1 + 1e-4) + 1e-5 * ref.abs()
        else:
            bound = bound + 2.0 ** -8 * ref.abs()
        assert bool(((got - ref).abs() <= bound + 1e-12).all())
        want = v[s * n:(s + 1) * n].float()
        if cdt == sp.SP_E4M3:
            q, sc = quantise(want)
            assert torch.equal(cache.codes(s, lens[s] + n, "v")[lens[s]:], q.view(torch.uint8))
        else:
            assert torch.equal(cache.values(s, lens[s] + n, "v")[lens[s]:], want.to(torch.bfloat16).double())


def test_append_takes_a_path_through_a_tree_by_id_with_strided_rows(torch):
    hkv, dh, N = 2, 128, 8
    wide = 5 * hkv * dh
    g = torch.Generator().manual_seed(2)
    buf = torch.randn((3 * N, wide), generator=g).to(torch.bfloat16).cuda()
    cache = Cache(sp.SP_E4M3, hkv, dh, [30, 30, 30, 30], 16)
    take = [[0, 2, 5], [1, 7, 7], [3, 0, 0]]
    rows = make_rows(torch, [3, 2, 0], 3, 3 * N, row0=[0, N, 2 * N], take=take, ks=wide, vs=wide)
    ids = torch.tensor([2, 0, 3], dtype=torch.int32).cuda()
    kp, vp = buf.data_ptr() + 2 * 2 * hkv * dh, buf.data_ptr() + 2 * 3 * hkv * dh
    assert append(torch, cache, [4, 9, 20, 0], rows, sp.SP_BF16, kp, vp, ids=ids, batch=3) == 0
    for b, (s, L, n) in enumerate([(2, 20, 3), (0, 4, 2)]):
        for which, first in (("k", 2), ("v", 3)):
            x = buf[[b * N + j for j in take[b][:n]], first * hkv * dh:(first + 1) * hkv * dh].float().cpu()
            q, _ = quantise(x.view(n, hkv, dh))
            assert torch.equal(cache.codes(s, L + n, which)[L:], q.view(torch.uint8))


def test_non_finite_elements_become_nan_and_leave_their_row_alone(torch):
    hkv, dh = 1, 64
    x = torch.randn((4, hkv, dh), generator=torch.Generator().manual_seed(1))
    x[1, 0, 5], x[2, 0, 0], x[2, 0, 63] = float("nan"), float("inf"), float("-inf")
    x[3] = 3e38
    cache = Cache(sp.SP_E4M3, hkv, dh, [8], 0)
    assert append(torch, cache, [0], make_rows(torch, None, 4, 4), sp.SP_F32, x.cuda(), x.cuda()) == 0
    got, fin = cache.values(0, 4, "v"), torch.isfinite(x)
    assert bool(torch.isnan(got[~fin]).all()) and bool(torch.isfinite(got[fin]).all())
    q, _ = quantise(x)
    assert torch.equal(cache.codes(0, 4, "k")[fin], q.view(torch.uint8)[fin])


def test_append_reports_what_it_cannot_place(torch):
    hkv, dh = 1, 128
    k = torch.ones((8, hkv, dh), dtype=torch.bfloat16).cuda()

    def fresh():
        return Cache(sp.SP_BF16, hkv, dh, [40, 40], 16, junk=3.0)

    c = fresh()  # past max_seq_len
    assert append(torch, c, [38, 0], make_rows(torch, None, 4, 8), sp.SP_BF16, k, k) == sp.SP_DEV_BAD_LENGTH
    assert bool((c.values(0, 40, "k")[38:] == 1).all()) and bool((c.values(0, 40, "k")[:38] == 3).all())
    c = fresh()  # no page
    c.table[1, 0] = 10 ** 6
    c.describe()
    assert append(torch, c, [0, 0], make_rows(torch, None, 4, 8), sp.SP_BF16, k, k) == sp.SP_DEV_BAD_PAGE
    c = fresh()  # rows outside the buffer
    assert append(torch, c, [0, 0], make_rows(torch, None, 4, 6), sp.SP_BF16, k, k) == sp.SP_DEV_BAD_ROW
    assert bool((c.values(1, 4, "k")[:2] == 1).all()) and bool((c.values(1, 4, "k")[2:] == 3).all())
    assert append(torch, c, [0, 0], make_rows(torch, [-1, 9], 4, 8), sp.SP_BF16, k, k) == sp.SP_DEV_BAD_ROW
    c = fresh()  # an id outside the cache, a length outside its bound
    ids = torch.tensor([0, 7], dtype=torch.int32).cuda()
    assert append(torch, c, [0, 0], make_rows(torch, None, 4, 8), sp.SP_BF16, k, k, ids=ids, batch=2) == sp.SP_DEV_BAD_SEQ_ID
    assert append(torch, c, [-3, 0], make_rows(torch, None, 4, 8), sp.SP_BF16, k, k) == sp.SP_DEV_BAD_LENGTH


@pytest.mark.parametrize("cdt", [sp.SP_E4M3, sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("dtype", [sp.SP_BF16, sp.SP_F32])
@pytest.mark.parametrize("page", LAYOUTS)
@pytest.mark.parametrize("dh", [128, 32])
def test_read_returns_the_values_and_zeros_past_the_end(torch, cdt, dtype, page, dh):
    lens, hkv, most = [0, 1, 33, 90], 2, 70
    g = torch.Generator().manual_seed(page)
    cache = Cache(cdt, hkv, dh, [x + 1 for x in lens], page)
    for s, n in enumerate(lens):
        cache.put(s, 0, torch.randn((n, hkv, dh), generator=g), torch.randn((n, hkv, dh), generator=g))
    k, v = (torch.full((4, most, hkv, dh), 9.0).to(torch_type(dtype)).cuda() for _ in range(2))
    first = torch.tensor([0, 0, 3, 30], dtype=torch.int32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = make_rows(torch, [most, 5, most, most], most, 4 * most)
    sp.sp_cache_read(torch.cuda.current_stream(), cache.desc, 4, None, torch.tensor(lens, dtype=torch.int32).cuda(),
                     first, rows, dtype, k, v, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for s, (f, n) in enumerate(zip([0, 0, 3, 30], [most, 5, most, most])):
        for out, which in ((k, "k"), (v, "v")):
            x = cache.values(s, lens[s], which)[f:f + n]
            want = torch.zeros((n, hkv, dh), dtype=torch.float64)
            want[:len(x)] = x
            # a code times its scale is one fp32 rounding of the float64 product, then bf16's
            assert torch.equal(out[s, :n].cpu(), want.float().to(out.dtype))
            assert bool((out[s, n:] == 9).all())


def test_read_takes_tokens_by_index(torch):
    cache = Cache(sp.SP_BF16, 1, 64, [50], 16)
    x = torch.arange(50.0)[:, None, None].expand(50, 1, 64).contiguous()
    cache.put(0, 0, x, -x)
    k, v = (torch.zeros((4, 1, 64), device="cuda") for _ in range(2))
    rows = make_rows(torch, None, 4, 4, take=[[7, 0, 49, 60]])
    sp.sp_cache_read(torch.cuda.current_stream(), cache.desc, 1, None, torch.tensor([50], dtype=torch.int32).cuda(), None,
                     rows, sp.SP_F32, k, v)
    torch.cuda.synchronize()
    assert k[:, 0, 0].tolist() == [7.0, 0.0, 49.0, 0.0] and v[:, 0, 5].tolist() == [-7.0, 0.0, -49.0, 0.0]


def test_what_is_appended_is_what_the_classify_attention_reads(torch):
    """sp_attend over a bf16 cache written by sp_cache_append equals sp_attend over the
    same cache written by the test."""
    hkv, dh, lens = 2, 128, [70, 33]
    g = torch.Generator().manual_seed(8)
    a, b = Cache(sp.SP_BF16, hkv, dh, [80, 40], 16, junk=0.0), Cache(sp.SP_BF16, hkv, dh, [80, 40], 16, junk=0.0)
    k, v = (torch.randn((103, hkv, dh), generator=g).to(torch.bfloat16) for _ in range(2))
    rows = make_rows(torch, lens, 70, 103, row0=[0, 70])
    assert append(torch, a, [0, 0], rows, sp.SP_BF16, k.cuda(), v.cuda()) == 0
    b.put(0, 0, k[:70].float(), v[:70].float())
    b.put(1, 0, k[70:].float(), v[70:].float())
    q, kn, vn = (torch.randn((2, 3, h, dh), generator=g).cuda() for h in (4, 2, 2))
    dims = sp.sp_attn_dims(4, 2, dh, 3, sp.SP_BF16, 100, 0, 0)
    ws = torch.empty(sp.sp_attend_workspace_bytes(dims, 2), dtype=torch.uint8, device="cuda")
    outs = []
    for c in (a, b):
        out = torch.empty((2, 3, 4, dh), device="cuda")
        sp.sp_attend(torch.cuda.current_stream(), dims, 2, None, torch.tensor(lens, dtype=torch.int32).cuda(), c.desc.kv,
                     q, kn, vn, out, sp.SP_F32, ws, ws.numel())
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(*outs)
