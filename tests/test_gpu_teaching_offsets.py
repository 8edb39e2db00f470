"""The teaching calls where offsets pass 32 bits, batches fill the tensor-core kernel's tables, and calls
run at once on streams of their own."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_norm import back64, norm64
from test_gpu_tree_backward import Case
from test_gpu_vocab_loss import backward, dims_of, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def test_norm_of_more_than_2_31_elements(torch):
    n, d = 530000, 4096  # 2.17e9
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 50000):
        x[i:i + 50000] = torch.randn(x[i:i + 50000].shape, generator=g, device="cuda")
    y = torch.empty_like(x)
    dims = sp.sp_norm_dims(n, d, sp.SP_BF16, sp.SP_BF16, 1e-6, 0, 0, 0, 0)
    sp.sp_norm(torch.cuda.current_stream(), dims, x, None, None, None, y)
    for at in (0, n // 2, n - 50):
        want = norm64(torch, x[at:at + 50], None, None, 1e-6)[1]
        assert bool(((y[at:at + 50].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -19)).all())
    dx = torch.empty_like(x)
    sp.sp_norm_backward(torch.cuda.current_stream(), dims, y, x, None, None, dx)
    for at in (0, n // 2, n - 50):
        want, size, _, _ = back64(torch, y[at:at + 50], x[at:at + 50], None, None, 1e-6)
        assert bool(((dx[at:at + 50].double() - want).abs() <= size * 2.0 ** -18 + want.abs() * 2.0 ** -8).all())


def test_a_head_of_more_than_2_31_elements(torch):
    n, d, V = 5, 4096, 530000  # 2.17e9 elements of W and of its gradient
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty((V, d), dtype=torch.bfloat16, device="cuda")
    for i in range(0, V, 50000):
        w[i:i + 50000] = torch.randn(w[i:i + 50000].shape, generator=g, device="cuda") * 0.02
    h = torch.randn((n, d), generator=g, device="cuda").to(torch.bfloat16)
    t = torch.tensor([0, V - 1, 300000, V - 2, 524290], dtype=torch.int32, device="cuda")
    dims = dims_of(h, w, d, sp.SP_BF16, 2)
    loss, lse, _ = forward(torch, dims, h, w, t)
    logits = torch.cat([h.double() @ w[i:i + 50000].double().T for i in range(0, V, 50000)], 1)
    want = torch.logsumexp(logits, -1)
    # logits of size 6 from 4096 products of sum |h w| 55 at most: 4100 steps of 2^-22 of it
    off = 55 * 4100 * 2.0 ** -22 + 2.0 ** -16
    assert bool(((lse.double() - want).abs() <= off).all())
    assert bool(((loss.double() - (want - logits[torch.arange(n), t.long()])).abs() <= 2 * off).all())
    dh, dw, _ = backward(torch, dims, h, w, t, lse, None)
    p = torch.softmax(logits, -1)
    p[torch.arange(n), t.long()] -= 1
    for v in (0, 300000, 524290, V - 2, V - 1):
        exact = p[:, v] @ h.double()
        lim = p[:, v].abs() @ h.double().abs() * (2 * off + 2.0 ** -7) + exact.abs() * 2.0 ** -8
        assert bool(((dw[v].double() - exact).abs() <= lim).all()), v
    exact = sum(p[:, i:i + 50000] @ w[i:i + 50000].double() for i in range(0, V, 50000))
    size = sum(p[:, i:i + 50000].abs() @ w[i:i + 50000].double().abs() for i in range(0, V, 50000))
    assert bool(((dh.double() - exact).abs() <= size * (2 * off + 2.0 ** -7) + exact.abs() * 2.0 ** -8).all())


@pytest.mark.parametrize("cdt,dtype", [(sp.SP_BF16, sp.SP_BF16), (sp.SP_F32, sp.SP_F32), (sp.SP_E4M3, sp.SP_BF16)])
def test_pages_behind_2_31_elements(torch, cdt, dtype):
    c = Case(torch, cdt, dtype, 16, 128, 4, 2, [100, 37], 3, seed=21)
    small = c.cache
    pages = 530000  # of 4096 elements
    for name in ("k", "v") + (("ks", "vs") if cdt == sp.SP_E4M3 else ()):  # (an 8-bit cache's scales with its pages)
        old = getattr(small, name)
        big = torch.zeros((pages,) + tuple(old.shape[1:]), dtype=old.dtype, device="cuda")
        big[pages - len(old):] = old
        setattr(small, name, big)
    small.table[small.table >= 0] += pages - small.n_pages
    small.n_pages = pages
    small.describe()
    c.check()


@pytest.mark.parametrize("cdt,hq,N", [(sp.SP_BF16, 2, 2), (sp.SP_E4M3, 2, 2), (sp.SP_E4M3, 16, 9)])
def test_a_batch_that_fills_the_tables(torch, cdt, hq, N):
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 2048).tolist()
    c = Case(torch, cdt, sp.SP_BF16, 16, 128, hq, 1, lens, N, path=2, seed=22)
    grads = c.forward().backward()
    assert c.status == 0
    for b in (0, 1, 777, 1500, 2046, 2047):
        want, lim, _, _ = c.reference(b)
        for g, w, m in zip(grads, want, lim):
            got = g.view(2048, N, -1)[b].cpu().double().view(w.shape)
            assert bool(((got - w).abs() <= m).all())


def test_calls_at_once_on_streams_of_their_own(torch):
    attend = [Case(torch, sp.SP_BF16, sp.SP_BF16, 16, 128, 8, 2, [900, 30, 2000], 6, seed=s).forward() for s in (30, 31)]
    want = [c.backward() for c in attend]
    losses = []
    for s in (32, 33):
        h, w, t, gl = inputs(torch, 300, 256, 3000, sp.SP_BF16, s, skip=0.2)
        dims = dims_of(h, w, 256, sp.SP_BF16, 0)
        loss, lse, _ = forward(torch, dims, h, w, t)
        losses.append((dims, h, w, t, lse, gl) + backward(torch, dims, h, w, t, lse, gl)[:2])
    streams = [torch.cuda.Stream() for _ in range(4)]
    ws = [torch.empty(sp.sp_attend_tree_backward_workspace_bytes(c.dims, c.cache.desc, 3), dtype=torch.uint8, device="cuda")
          for c in attend]
    ws += [torch.empty(sp.sp_vocab_loss_backward_workspace_bytes(x[0]), dtype=torch.uint8, device="cuda") for x in losses]
    out = [[torch.zeros_like(x) for x in w] for w in want] + [[torch.zeros_like(x) for x in l[6:]] for l in losses]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, c in enumerate(attend):
            sp.sp_attend_tree_backward(streams[i], c.dims, c.cache.desc, 3, None, c.lens_d, c.mask_d, c.n_d, *c.rows, c.out,
                                       c.lse, c.do_d, *out[i], ws[i], ws[i].numel())
        for i, (dims, h, w, t, lse, gl, _, _) in enumerate(losses):
            sp.sp_vocab_loss_backward(streams[2 + i], dims, h, w, t, lse, gl, *out[2 + i], ws[2 + i], ws[2 + i].numel())
    torch.cuda.synchronize()
    for got, exact in zip(out, want + [l[6:] for l in losses]):
        assert all(torch.equal(x, y) for x, y in zip(got, exact))


def test_sequences_by_id_and_one_id_twice(torch):
    c = Case(torch, sp.SP_BF16, sp.SP_BF16, 16, 128, 4, 2, [300, 70, 5], 4, seed=34)
    a = c.forward().backward()
    # the same calls through ids: entry i of the batch is sequence ids[i]; both may be one
    ids = torch.tensor([0, 0, 2], dtype=torch.int32, device="cuda")
    size = sp.sp_attend_tree_backward_workspace_bytes(c.dims, c.cache.desc, 3)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    rows = [x.view(3, 4, -1).clone() for x in c.rows + [c.out, c.lse, c.do_d]]
    for x in rows:
        x[1] = x[0]
    mask = c.mask_d.clone()
    mask[1] = mask[0]
    grads = [torch.zeros_like(x) for x in a]
    sp.sp_attend_tree_backward(torch.cuda.current_stream(), c.dims, c.cache.desc, 3, ids, c.lens_d, mask, None, *rows, *grads, ws,
                               size)
    torch.cuda.synchronize()
    for x, y in zip(grads, a):
        x, y = x.view(3, 4, -1), y.view(3, 4, -1)
        # (shares are cut elsewhere: sums of other parts; the first two are each other's equals to a rounding)
        assert bool(((x[0].float() - y[0].float()).abs() <= y[0].float().abs() * 2.0 ** -7 + 2.0 ** -9 * y[0].float().abs().max()).all())
        assert bool(((x[0].float() - x[1].float()).abs() <= x[0].float().abs() * 2.0 ** -7 + 2.0 ** -9 * x[0].float().abs().max()).all())
        assert bool(((x[2].float() - y[2].float()).abs() <= y[2].float().abs() * 2.0 ** -7 + 2.0 ** -9 * y[2].float().abs().max()).all())


def test_calls_in_a_row_that_share_a_workspace(torch):
    # nothing waits between them: a kernel that ran ahead would meet another call's data
    st = torch.cuda.Stream()
    cases = [Case(torch, sp.SP_BF16, sp.SP_BF16, 16, 128, 8, 2, lens, 6, seed=40 + i).forward()
             for i, lens in enumerate(([900, 30, 2000], [3, 0, 400]))]
    want = [c.backward() for c in cases]
    ws = torch.empty(max(sp.sp_attend_tree_backward_workspace_bytes(c.dims, c.cache.desc, 3) for c in cases), dtype=torch.uint8,
                     device="cuda")
    outs = [[torch.zeros_like(x) for x in want[i % 2]] for i in range(10)]
    losses = []
    for s in (42, 43):
        h, w, t, gl = inputs(torch, 200 if s == 42 else 40, 128, 2500, sp.SP_BF16, s, skip=0.2)
        dims = dims_of(h, w, 128, sp.SP_BF16, 0)
        loss, lse, _ = forward(torch, dims, h, w, t)
        losses.append((dims, h, w, t, gl, loss, lse) + backward(torch, dims, h, w, t, lse, gl)[:2])
    wl = torch.empty(max(sp.sp_vocab_loss_backward_workspace_bytes(x[0]) for x in losses), dtype=torch.uint8, device="cuda")
    found = [[torch.zeros_like(x) for x in losses[i % 2][5:]] for i in range(10)]
    torch.cuda.synchronize()
    for i in range(10):
        c = cases[i % 2]
        sp.sp_attend_tree_backward(st, c.dims, c.cache.desc, 3, None, c.lens_d, c.mask_d, c.n_d, *c.rows, c.out, c.lse, c.do_d,
                                   *outs[i], ws, ws.numel())
        dims, h, w, t, gl = losses[i % 2][:5]
        loss, lse, dh, dw = found[i]
        sp.sp_vocab_loss(st, dims, h, w, t, loss, lse, wl, wl.numel())
        sp.sp_vocab_loss_backward(st, dims, h, w, t, lse, gl, dh, dw, wl, wl.numel())
    st.synchronize()
    for i in range(10):
        assert all(torch.equal(x, y) for x, y in zip(outs[i], want[i % 2]))
        assert all(torch.equal(x, y) for x, y in zip(found[i], losses[i % 2][5:]))
