"""Row norms and their backward pass against float64 from the definitions."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu
HALF = {sp.SP_F32: 2.0 ** -24, sp.SP_BF16: 2.0 ** -8, sp.SP_E4M3: 2.0 ** -4}  # a rounding, relative
EPS = 1e-6


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def rows(torch, g, n, d, dtype, stride=0, std=1.0, at=0):
    """n rows of d, `stride` elements apart (0: d), `at` elements into their buffer; NaN between them."""
    stride = stride or d
    buf = torch.full((n * stride + at + 8,), float("nan")).to(torch_type(dtype)).cuda()
    view = buf[at:at + n * stride].view(n, stride)[:, :d]
    view.copy_((torch.randn((n, d), generator=g) * std).to(torch_type(dtype)))
    return view


def norm64(torch, x, r, gain, eps):
    s = x.double() + (r.double() if r is not None else 0.0)
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s, y * gain.double() if gain is not None else y


def dims_of(n, d, dtype, out, eps, x, r, s, y):
    return sp.sp_norm_dims(n, d, dtype, out, eps, *(0 if t is None else t.stride(0) for t in (x, r, s, y)))


def check(torch, n, d, dtype, out, residual=True, gain=True, want_sum=True, strides=(0, 0, 0, 0), at=0, std=1.0, eps=EPS,
          seed=0):
    g = torch.Generator().manual_seed(seed)
    x = rows(torch, g, n, d, dtype, strides[0], std, at)
    r = rows(torch, g, n, d, dtype, strides[1], std, at) if residual else None
    w = (1 + 0.2 * torch.randn(d, generator=g)).cuda() if gain else None
    s = rows(torch, g, n, d, dtype, strides[2], at=at) if want_sum else None
    y = rows(torch, g, n, d, dtype, strides[3], at=at) if out != sp.SP_E4M3 else torch.zeros(
        (n, strides[3] or d), dtype=torch.float8_e4m3fn, device="cuda")[:, :d]
    scale = torch.full((n,), float("nan"), device="cuda") if out == sp.SP_E4M3 else None
    sp.sp_norm(torch.cuda.current_stream(), dims_of(n, d, dtype, out, eps, x, r, s, y), x, r, w, s, y, scale)
    torch.cuda.synchronize()
    s64, y64 = norm64(torch, x, r, w, eps)
    if want_sum:
        assert bool(((s.double() - s64).abs() <= s64.abs() * (HALF[dtype] + 2.0 ** -23)).all())
    # fp32: the sum s, its squares' sum (rows of up to 2^13 elements in 32-wide trees), rsqrt, two products
    rel = 2.0 ** -19 + HALF[out]
    if out == sp.SP_E4M3:
        amax = y64.abs().amax(-1).clamp_min(2.0 ** -60)
        assert bool(((scale.double() - amax / 448).abs() <= amax / 448 * 2.0 ** -18).all())
        got = y.float().double() * scale.double()[:, None]
        lim = y64.abs() * rel + amax[:, None] / 448 * 2.0 ** -10  # (below 2^-6 the codes are 2^-9 apart)
    else:
        got, lim = y.double(), y64.abs() * rel + 1e-38
    assert bool(((got - y64).abs() <= lim).all()), float(((got - y64).abs() / lim).max())


TYPES = [(sp.SP_F32, sp.SP_F32), (sp.SP_BF16, sp.SP_BF16), (sp.SP_F32, sp.SP_E4M3), (sp.SP_BF16, sp.SP_E4M3)]


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("d", [1, 7, 8, 40, 128, 256, 264, 1000, 1024, 2560, 4096, 5120, 8200, 20000, 40000])
def test_lengths(torch, dtype, out, d):
    check(torch, 7, d, dtype, out, seed=d)


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("residual,gain,want_sum", [(False, True, False), (False, False, True), (True, True, False)])
def test_parts_left_out(torch, dtype, out, residual, gain, want_sum):
    check(torch, 33, 512, dtype, out, residual, gain, want_sum)


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("strides,at", [((1024, 1032, 1040, 1048), 0), ((1001, 0, 1003, 1005), 0), ((0, 0, 0, 0), 1),
                                        ((1008, 0, 0, 1001), 0)])
def test_strides_and_alignment(torch, dtype, out, strides, at):
    check(torch, 5, 1000, dtype, out, strides=strides, at=at)


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("n", [1, 2, 5, 1000, 70001])
def test_row_counts(torch, dtype, out, n):
    check(torch, n, 64, dtype, out, seed=n)


@pytest.mark.parametrize("d", [96, 100, 4096, 40000])
@pytest.mark.parametrize("std,eps", [(1e25, EPS), (1e37, EPS), (1e-25, 0.0), (1e-37, 0.0), (1e-25, EPS)])
def test_rows_whose_squares_leave_fp32(torch, d, std, eps):
    check(torch, 3, d, sp.SP_F32, sp.SP_F32, residual=False, want_sum=False, std=std, eps=eps)


@pytest.mark.parametrize("d", [64, 100, 2560])
def test_zero_rows_and_non_finite_elements(torch, d):
    x = torch.zeros((4, d), device="cuda")
    x[1, 3], x[2, 5] = float("nan"), float("inf")
    x[3] = 1.0
    for out in (sp.SP_F32, sp.SP_E4M3):
        y = torch.empty((4, d), dtype=torch_type(out), device="cuda")
        scale = torch.empty(4, device="cuda")
        sp.sp_norm(torch.cuda.current_stream(), sp.sp_norm_dims(4, d, sp.SP_F32, out, EPS, 0, 0, 0, 0), x, None, None, None,
                   y, scale)
        y = y.float()
        assert bool((y[0] == 0).all()) and bool(y[1].isnan().all()) and bool(y[2, 5].isnan())
        assert bool((y[2, :5] == 0).all()) and bool(y[3].isfinite().all())


@pytest.mark.parametrize("d", [64, 100])
def test_in_place(torch, d):
    g = torch.Generator().manual_seed(1)
    x, r = rows(torch, g, 9, d, sp.SP_BF16), rows(torch, g, 9, d, sp.SP_BF16)
    want_s, want_y = x.clone(), x.clone()
    dims = sp.sp_norm_dims(9, d, sp.SP_BF16, sp.SP_BF16, EPS, 0, 0, 0, 0)
    sp.sp_norm(torch.cuda.current_stream(), dims, x, r, None, want_s, want_y)
    sp.sp_norm(torch.cuda.current_stream(), dims, x, r, None, r, x)
    assert torch.equal(r, want_s) and torch.equal(x, want_y)


def back64(torch, dy, s, gain, ds, eps):
    dy, s = dy.double(), s.double()
    w = gain.double() if gain is not None else torch.ones(s.shape[1], dtype=torch.float64, device=s.device)
    rstd = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    xh = s * rstd
    dx = rstd * (w * dy - xh * (w * dy * xh).mean(-1, keepdim=True))
    size = rstd * ((w * dy).abs() + xh.abs() * (w * dy * xh).abs().mean(-1, keepdim=True))
    return dx + (ds.double() if ds is not None else 0.0), size, (dy * xh).sum(0), (dy * xh).abs().sum(0)


def back(torch, n, d, dtype, beside=True, gain=True, want_gain=True, strides=(0, 0, 0, 0), at=0, std=1.0, seed=0, eps=EPS):
    g = torch.Generator().manual_seed(seed)
    s, dy = rows(torch, g, n, d, dtype, strides[2], std, at), rows(torch, g, n, d, dtype, strides[3], 0.1, at)
    ds = rows(torch, g, n, d, dtype, strides[1], 0.1, at) if beside else None
    w = (1 + 0.2 * torch.randn(d, generator=g)).cuda() if gain else None
    dx = rows(torch, g, n, d, dtype, strides[0], at=at)
    dims = dims_of(n, d, dtype, dtype, eps, dx, ds, s, dy)
    size = sp.sp_norm_backward_workspace_bytes(dims)
    ws = torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda")
    dg = torch.full((d,), float("nan"), device="cuda") if want_gain else None
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, dy, s, w, ds, dx, dg, ws if want_gain else None, size)
    torch.cuda.synchronize()
    want, mag, wg, wga = back64(torch, dy, s, w, ds, eps)
    lim = mag * 2.0 ** -18 + want.abs() * (HALF[dtype] + 2.0 ** -23) + 1e-38
    assert bool(((dx.double() - want).abs() <= lim).all()), float(((dx.double() - want).abs() / lim).max())
    if want_gain:  # n products, added in runs and then the runs: fewer than n + 64 roundings; xh 2^-19
        assert bool(((dg.double() - wg).abs() <= wga * ((n + 64) * 2.0 ** -24 + 2.0 ** -19) + 1e-38).all())
    return dx, dg


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("d", [1, 7, 8, 128, 264, 1000, 2560, 4096, 8200, 20000, 40000])
def test_backward_lengths(torch, dtype, d):
    back(torch, 11, d, dtype, seed=d)


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("n", [1, 2, 700, 5003])
@pytest.mark.parametrize("beside,gain,want_gain", [(True, True, True), (False, True, False), (False, False, True)])
def test_backward_row_counts_and_parts(torch, dtype, n, beside, gain, want_gain):
    back(torch, n, 192, dtype, beside, gain, want_gain, seed=n)


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("strides,at", [((1024, 1032, 1040, 1048), 0), ((1001, 0, 1003, 1005), 0), ((0, 0, 0, 0), 1)])
def test_backward_strides(torch, dtype, strides, at):
    back(torch, 300, 1000, dtype, strides=strides, at=at)


@pytest.mark.parametrize("d", [96, 100, 4096])
@pytest.mark.parametrize("std,eps", [(1e25, EPS), (1e-25, 0.0), (1e-25, EPS)])
def test_backward_out_of_range(torch, d, std, eps):
    back(torch, 3, d, sp.SP_F32, std=std, eps=eps, beside=False)


def test_backward_repeats_its_bits_and_works_in_place(torch):
    dx, dg = back(torch, 3000, 1024, sp.SP_BF16)
    again, dg2 = back(torch, 3000, 1024, sp.SP_BF16)
    assert torch.equal(dx, again) and torch.equal(dg, dg2)
    for d in (64, 100):
        g = torch.Generator().manual_seed(2)
        s, dy, ds = (rows(torch, g, 9, d, sp.SP_F32) for _ in range(3))
        dims = sp.sp_norm_dims(9, d, sp.SP_F32, sp.SP_F32, EPS, 0, 0, 0, 0)
        want = torch.empty_like(s)
        sp.sp_norm_backward(torch.cuda.current_stream(), dims, dy, s, None, ds, want)
        for i in range(3):
            a = [dy.clone(), s.clone(), ds.clone()]
            sp.sp_norm_backward(torch.cuda.current_stream(), dims, a[0], a[1], None, a[2], a[i])
            assert torch.equal(a[i], want)


def test_backward_of_no_rows_clears_the_gain(torch):
    dims = sp.sp_norm_dims(0, 64, sp.SP_F32, sp.SP_F32, EPS, 0, 0, 0, 0)
    dg = torch.ones(64, device="cuda")
    size = sp.sp_norm_backward_workspace_bytes(dims)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, None, None, None, None, None, dg, ws, size)
    assert bool((dg == 0).all())


def test_backward_against_differences(torch):
    # the slope of sum(dy y) + sum(ds s) along a direction, from the forward formula in float64:
    # h = 1e-4 leaves h^2 / 6 of third derivatives (of size 1), fp32 gradients 2^-17 of their terms
    n, d = 6, 200
    g = torch.Generator().manual_seed(3)
    s, dy, ds = (torch.randn((n, d), generator=g).cuda() for _ in range(3))
    w, u = (1 + 0.2 * torch.randn(d, generator=g)).cuda(), torch.randn((n, d), generator=g).cuda()
    dims = sp.sp_norm_dims(n, d, sp.SP_F32, sp.SP_F32, EPS, 0, 0, 0, 0)
    dx = torch.empty_like(s)
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, dy, s, w, ds, dx)
    f = lambda t: (norm64(torch, s.double() + t * u.double(), None, w, EPS)[1] * dy.double()).sum() + (  # noqa: E731
        (s.double() + t * u.double()) * ds.double()).sum()
    slope, got = float((f(1e-4) - f(-1e-4)) / 2e-4), float((dx.double() * u.double()).sum())
    assert abs(slope - got) <= 1e-6 * n * d
