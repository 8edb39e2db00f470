"""Cross entropy over a vocabulary and its gradients against float64 from the definitions."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from token_cache_util import torch_type

pytestmark = pytest.mark.gpu
HALF = {sp.SP_F32: 2.0 ** -24, sp.SP_BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def inputs(torch, n, d, V, dtype, seed, skip=0.0, std=1.0, hs=0, ws=0):
    g = torch.Generator().manual_seed(seed)
    t = torch_type(dtype)
    h = torch.full((n, hs or d), float("nan")).to(t)
    w = torch.full((V, ws or d), float("nan")).to(t)
    h[:, :d] = torch.randn((n, d), generator=g).to(t)
    w[:, :d] = (torch.randn((V, d), generator=g) * std * 2.0 / d ** 0.5).to(t)
    targets = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    targets[torch.rand(n, generator=g) < skip] = -1
    gl = torch.rand(n, generator=g) + 0.1
    return h.cuda(), w.cuda(), targets.cuda(), gl.cuda()


def dims_of(h, w, d, dtype, path):
    return sp.sp_vocab_dims(h.shape[0], w.shape[0], d, dtype, path, h.stride(0), w.stride(0))


def forward(torch, dims, h, w, t, stream=None):
    size = sp.sp_vocab_loss_workspace_bytes(dims)
    assert size > 0, sp.sp_last_error()
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # scratch holds NaN
    loss, lse = (torch.full((dims.n_tokens,), float("nan"), device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    sp.sp_vocab_loss(stream or torch.cuda.current_stream(), dims, h, w, t, loss, lse, ws, size, status)
    torch.cuda.synchronize()
    return loss, lse, int(status)


def backward(torch, dims, h, w, t, lse, gl, head=True, stream=None):
    size = sp.sp_vocab_loss_backward_workspace_bytes(dims)
    assert size > 0, sp.sp_last_error()
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    dh, dw = torch.full_like(h, float("nan")), torch.full_like(w, float("nan")) if head else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    sp.sp_vocab_loss_backward(stream or torch.cuda.current_stream(), dims, h, w, t, lse, gl, dh, dw, ws, size, status)
    torch.cuda.synchronize()
    return dh, dw, int(status)


def check(torch, n, d, V, dtype, path=0, skip=0.0, std=1.0, head=True, hs=0, ws=0, seed=0, ones=False, junk=True):
    h, w, t, gl = inputs(torch, n, d, V, dtype, seed, skip, std, hs, ws)
    if junk:  # a token without a target is not looked at
        h[t < 0] = float("nan")
    dims = dims_of(h, w, d, dtype, path)
    tensor = dtype == sp.SP_BF16 and path != 1 and not (d % 8 or h.stride(0) % 8 or w.stride(0) % 8)
    loss, lse, status = forward(torch, dims, h, w, t)
    assert status == 0
    keep = (t >= 0).nonzero()[:, 0]
    hot = (torch.arange(len(keep), device="cuda"), t[keep].long())
    x, y = h[keep, :d].double(), w[:, :d].double()
    logits = x @ y.T
    # a logit: d products added in fp32 (2^-22 a step for the tensor cores' sums)
    off = (x.abs() @ y.abs().T).amax(-1) * (d + 4) * (2.0 ** -22 if tensor else 2.0 ** -24)
    want = torch.logsumexp(logits, -1)
    # the sum: V terms in fp32 trees of 128 and 256 or serial runs of V / 64 / 32, logarithms to 2^-22 of their size
    lim = off + 2.0 ** -17 + want.abs() * 2.0 ** -21
    assert bool(((lse[keep].double() - want).abs() <= lim).all()), float(((lse[keep].double() - want).abs() / lim).max())
    exact = want - logits[hot]
    lim = 2 * off + 2.0 ** -17 + (want.abs() + logits[hot].abs()) * 2.0 ** -21
    assert bool(((loss[keep].double() - exact).abs() <= lim).all())
    assert bool((loss[t < 0] == 0).all()) and bool((lse[t < 0] == 0).all())

    dh, dw, status = backward(torch, dims, h, w, t, lse, None if ones else gl, head)
    assert status == 0
    p = torch.softmax(logits, -1)
    up = (torch.ones_like(gl) if ones else gl)[keep].double()[:, None]
    q = p.clone()
    q[hot] -= 1.0
    q *= up
    # g: its weight moves by the errors of logit and log sum; p - 1 loses 2^-23 of 1; bf16 as an operand
    ge = p * up * (2 * off[:, None] + 2.0 ** -16 + want.abs()[:, None] * 2.0 ** -20)
    ge[hot] += up[:, 0] * 2.0 ** -23
    ge += q.abs() * (HALF[sp.SP_BF16] if tensor else 2.0 ** -22)
    half, step = HALF[dtype], 2.0 ** -22 if tensor else 2.0 ** -24
    want = q @ y
    lim = ge @ y.abs() + (q.abs() @ y.abs()) * min((V + 8) * step, 2.0 ** -12) + want.abs() * half + 1e-38
    got = dh[keep, :d].double()
    assert bool(((got - want).abs() <= lim).all()), float(((got - want).abs() / lim).max())
    assert bool((dh[t < 0][:, :d] == 0).all())
    if d < h.stride(0):
        assert bool(dh[:, d:].isnan().all())
    if head:
        want = q.T @ x
        lim = ge.T @ x.abs() + (q.T.abs() @ x.abs()) * (len(keep) + 8) * step + want.abs() * half + 1e-38
        got = dw[:, :d].double()
        assert bool(((got - want).abs() <= lim).all()), float(((got - want).abs() / lim).max())
        if d < w.stride(0):
            assert bool(dw[:, d:].isnan().all())


WAYS = [(sp.SP_F32, 1), (sp.SP_BF16, 1), (sp.SP_BF16, 2)]


@pytest.mark.parametrize("dtype,path", WAYS)
@pytest.mark.parametrize("n,d,V", [(1, 8, 1), (1, 8, 2), (2, 16, 3), (5, 64, 37), (3, 72, 256), (64, 128, 257), (130, 200, 511),
                                   (256, 64, 512), (257, 1032, 300), (300, 264, 1000), (33, 24, 5000), (1, 520, 2049)])
def test_sizes(torch, dtype, path, n, d, V):
    check(torch, n, d, V, dtype, path, seed=n + V)


@pytest.mark.parametrize("dtype,path", WAYS)
@pytest.mark.parametrize("skip", [0.3, 0.9, 1.0])
def test_tokens_without_a_target(torch, dtype, path, skip):
    check(torch, 300, 136, 700, dtype, path, skip=skip)


@pytest.mark.parametrize("dtype,path", WAYS)
def test_frozen_head_and_unit_gradients(torch, dtype, path):
    check(torch, 70, 128, 300, dtype, path, head=False)
    check(torch, 70, 128, 300, dtype, path, ones=True, skip=0.2)


@pytest.mark.parametrize("dtype,path", WAYS)
def test_strides(torch, dtype, path):
    check(torch, 40, 72, 300, dtype, path, hs=96, ws=80, skip=0.1)


@pytest.mark.parametrize("n,d,V", [(20, 7, 50), (20, 33, 50), (9, 1, 3)])
def test_rows_that_are_not_vectors(torch, n, d, V):
    check(torch, n, d, V, sp.SP_BF16)
    check(torch, n, d, V, sp.SP_F32)
    check(torch, n, 8 * d, V, sp.SP_BF16, hs=8 * d + 1, ws=8 * d + 3)


@pytest.mark.parametrize("dtype,path", WAYS)
def test_sharp_distributions(torch, dtype, path):
    check(torch, 50, 64, 400, dtype, path, std=20.0)


def test_a_vocabulary_in_pieces(torch):
    check(torch, 8003, 16, 20001, sp.SP_BF16, skip=0.1)
    check(torch, 3000, 8, 9000, sp.SP_F32)


def test_products_split_along_the_vocabulary(torch):
    check(torch, 10, 64, 30000, sp.SP_BF16)


@pytest.mark.parametrize("dtype,path", WAYS)
def test_targets_out_of_range_are_reported(torch, dtype, path):
    h, w, t, gl = inputs(torch, 9, 16, 40, dtype, 1)
    t[3], t[5] = 40, -7
    dims = dims_of(h, w, 16, dtype, path)
    loss, lse, status = forward(torch, dims, h, w, t)
    assert status == sp.SP_DEV_BAD_ROW and bool((loss[[3, 5]] == 0).all()) and bool(loss[[0, 8]].isfinite().all())
    dh, dw, status = backward(torch, dims, h, w, t, lse, gl)
    assert status == sp.SP_DEV_BAD_ROW and bool((dh[[3, 5]] == 0).all()) and bool(dw.isfinite().all())


@pytest.mark.parametrize("dtype,path", WAYS)
def test_non_finite_rows_stay_their_own(torch, dtype, path):
    h, w, t, gl = inputs(torch, 20, 64, 500, dtype, 2)
    h[4, 3] = float("nan")
    dims = dims_of(h, w, 64, dtype, path)
    loss, lse, _ = forward(torch, dims, h, w, t)
    others = [i for i in range(20) if i != 4]
    assert bool(loss[4].isnan()) and bool(loss[others].isfinite().all())
    dh, dw, _ = backward(torch, dims, h, w, t, lse, gl)
    assert bool(dh[4].isnan().all()) and bool(dh[others].isfinite().all()) and bool(dw.isnan().all())


@pytest.mark.parametrize("dtype,path", WAYS)
def test_no_tokens(torch, dtype, path):
    dims = sp.sp_vocab_dims(0, 30, 16, dtype, path, 0, 24)
    dw = torch.ones((30, 24), dtype=torch_type(dtype), device="cuda")
    sp.sp_vocab_loss(torch.cuda.current_stream(), dims, None, None, None, None, None, None, 0)
    sp.sp_vocab_loss_backward(torch.cuda.current_stream(), dims, None, None, None, None, None, None, dw, None, 0)
    assert bool((dw[:, :16] == 0).all()) and bool((dw[:, 16:] == 1).all())


@pytest.mark.parametrize("dtype,path", WAYS)
def test_the_same_bits_every_time_captured_too(torch, dtype, path):
    h, w, t, gl = inputs(torch, 200, 128, 3001, dtype, 3, skip=0.2)
    dims = dims_of(h, w, 128, dtype, path)
    loss, lse, _ = forward(torch, dims, h, w, t)
    dh, dw, _ = backward(torch, dims, h, w, t, lse, gl)
    a, b = sp.sp_vocab_loss_workspace_bytes(dims), sp.sp_vocab_loss_backward_workspace_bytes(dims)
    ws = torch.empty(max(a, b), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(x) for x in (loss, lse, dh, dw)]
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        sp.sp_vocab_loss(s, dims, h, w, t, out[0], out[1], ws, a)
        sp.sp_vocab_loss_backward(s, dims, h, w, t, out[1], gl, out[2], out[3], ws, b)
    for _ in range(2):
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, (loss, lse, dh, dw)))


def test_gradients_against_differences(torch):
    # the slope of sum(gl loss) along directions of h and w, from the loss formula in float64: h = 1e-4
    # leaves h^2 / 6 of third derivatives (below 40), fp32 gradients 2^-15 of their terms' sum
    n, d, V = 12, 40, 90
    h, w, t, gl = inputs(torch, n, d, V, sp.SP_F32, 4)
    dims = dims_of(h, w, d, sp.SP_F32, 0)
    _, lse, _ = forward(torch, dims, h, w, t)
    dh, dw, _ = backward(torch, dims, h, w, t, lse, gl)
    g = torch.Generator().manual_seed(5)
    u, z = torch.randn((n, d), generator=g).double().cuda() / d, torch.randn((V, d), generator=g).double().cuda() / d

    def f(a):
        x = (h.double() + a * u) @ (w.double() + a * z).T
        return float((gl.double() * (torch.logsumexp(x, -1) - x[torch.arange(n), t.long()])).sum())
    slope = (f(1e-4) - f(-1e-4)) / 2e-4
    got = float((dh.double() * u).sum() + (dw.double() * z).sum())
    size = float((dh.double() * u).abs().sum() + (dw.double() * z).abs().sum())
    assert abs(slope - got) <= size * 2.0 ** -15 + 1e-7
