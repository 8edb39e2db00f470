"""Norms of rows and of numbers of rows so long that a serial fp32 sum would show: equal terms are rounded the
same way at every step, so that errors add up instead of cancelling."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_norm import EPS, HALF
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu
# A thread's run of 16 terms, the runs and the threads in 64 bits, then one rounding, the root and two products
REL = 2.0 ** -19


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("dtype", [sp.SP_F32, sp.SP_BF16])
@pytest.mark.parametrize("d", [1 << 22, (1 << 22) + 3, 1 << 24])
@pytest.mark.parametrize("value", [0.7, 1.3])
def test_long_rows_of_equal_elements(torch, dtype, d, value):
    t = torch_type(dtype)
    x = torch.full((2, d), value, dtype=t, device="cuda")
    x[1] *= -3
    y = torch.empty_like(x)
    dims = sp.sp_norm_dims(2, d, dtype, dtype, EPS, 0, 0, 0, 0)
    sp.sp_norm(torch.cuda.current_stream(), dims, x, None, None, None, y)
    s = x[:, :1].double()
    want = s / torch.sqrt(s * s + EPS)
    err = (y.double() - want).abs() / (want.abs() * (REL + HALF[dtype]))
    assert float(err.max()) <= 1, float(err.max())
    # its backward pass: output gradients 1 and 2 in turn, mean xh g = 1.5 xh
    dy = torch.ones_like(x)
    dy[:, 1::2] = 2
    dx = torch.empty_like(x)
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, dy, x, None, None, dx)
    rstd = 1 / torch.sqrt(s * s + EPS)
    xh = s * rstd
    mean = (d // 2 * 2 + (d - d // 2)) / d
    for at, g in ((0, 1.0), (1, 2.0)):
        want = rstd * (g - xh * xh * mean)
        size = rstd * (g + xh * xh * mean)
        err = (dx[:, at::2].double() - want).abs() / (size * 2 * REL + want.abs() * HALF[dtype])
        assert float(err.max()) <= 1, (at, float(err.max()))


@pytest.mark.parametrize("dtype,d,n", [(sp.SP_F32, 64, 4000001), (sp.SP_BF16, 64, 4000001), (sp.SP_F32, 60, 1000003),
                                       (sp.SP_BF16, 1032, 500009), (sp.SP_F32, 1032, 500009)])
def test_gain_gradient_of_many_equal_rows(torch, dtype, d, n):
    # columns have output gradients of their own, every row is the same
    t = torch_type(dtype)
    g = torch.Generator().manual_seed(d)
    row, up = torch.randn(d, generator=g).to(t).cuda(), (1 + torch.rand(d, generator=g)).to(t).cuda()
    s, dy = row.expand(n, d).contiguous(), up.expand(n, d).contiguous()
    dx, dg = torch.empty_like(s), torch.full((d,), float("nan"), device="cuda")
    dims = sp.sp_norm_dims(n, d, dtype, dtype, EPS, 0, 0, 0, 0)
    size = sp.sp_norm_backward_workspace_bytes(dims)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # scratch holds NaN
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, dy, s, None, None, dx, dg, ws, size)
    xh = row.double() / torch.sqrt((row.double() ** 2).mean() + EPS)
    want = n * up.double() * xh
    # xh and its product 2^-19; runs of at most 208 rows (at most 20 here), walkers in 32 sums of at most 20
    # or with what the additions cut off, those in pairs: 208 + 20 + 20 + 5 < 255 roundings
    lim = want.abs() * (2.0 ** -19 + 255 * 2.0 ** -24)
    err = ((dg.double() - want).abs() / lim).max()
    print("worst", float(((dg.double() - want) / want).abs().max()))
    assert float(err) <= 1, float(err)
