"""Backward pass of the attention of trees over [cache ; tree], and the forward pass's log sums,
against float64 from the definitions, on every path."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_tree import fill, tree_call
from token_cache_util import Cache, mask_tensor, random_parents, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def as_rows(torch, x, stride):
    """x [rows][heads][dh] on the GPU in rows `stride` elements apart (0: dense), NaN between them."""
    x = x.flatten(0, -3).flatten(1)
    buf = torch.full((x.shape[0], stride or x.shape[1]), float("nan"), dtype=x.dtype, device="cuda")
    buf[:, :x.shape[1]] = x.cuda()
    return buf


class Case:
    """Inputs of a call, its forward pass and its reference."""

    def __init__(self, torch, cdt, dtype, page, dh, hq, hkv, lens, N, n_nodes=None, path=0, seed=0, scale=0.0, chain=False,
                 strides=(0, 0, 0), q_std=1.0, max_len=None):
        self.torch, self.lens, self.N, self.n_nodes, self.chain = torch, lens, N, n_nodes, chain
        self.dtype, self.hq, self.hkv, self.dh, self.path = dtype, hq, hkv, dh, path
        self.cache = Cache(cdt, hkv, dh, [max(x, 1) for x in lens], page, seed)
        if max_len is not None:
            self.cache.desc.max_seq_len = max_len
        g = fill(torch, self.cache, lens, seed)
        rng, B, t = np.random.default_rng(seed), len(lens), torch_type(dtype)
        self.q = (torch.randn((B, N, hq, dh), generator=g) * q_std).to(t)
        self.k, self.v = (torch.randn((B, N, hkv, dh), generator=g).to(t) for _ in range(2))
        self.do = torch.randn((B, N, hq, dh), generator=g).to(t)
        self.masks = np.stack([sp.sp_tree_masks(list(range(-1, N - 1)) if chain else random_parents(rng, N))[0]
                               for _ in range(B)])
        self.scale = scale or dh ** -0.5
        self.dims = sp.sp_tree_dims(hq, N, dtype, path, 0, scale, *strides)
        self.strides = strides
        self.tensor = dtype == sp.SP_BF16 and dh == 128 and cdt != sp.SP_F32 and path != 1

    def forward(self):
        torch, B = self.torch, len(self.lens)
        self.rows = [as_rows(torch, x, s) for x, s in zip((self.q, self.k, self.v), self.strides)]
        self.lens_d = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.n_d = None if self.n_nodes is None else torch.tensor(self.n_nodes, dtype=torch.int32).cuda()
        self.mask_d = None if self.chain else mask_tensor(torch, self.masks)
        size = sp.sp_attend_tree_workspace_bytes(self.dims, self.cache.desc, B)
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
        self.out = torch.full((B * self.N, self.hq, self.dh), float("nan")).to(torch_type(self.dtype)).cuda()
        self.lse = torch.full((B * self.N, self.hq), float("nan"), device="cuda")
        torch.cuda.synchronize()
        sp.sp_attend_tree_lse(torch.cuda.current_stream(), self.dims, self.cache.desc, B, None, self.lens_d, self.mask_d,
                              self.n_d, *self.rows, self.out, self.lse, ws, size)
        torch.cuda.synchronize()
        return self

    def backward(self, stream=None, grads=None, ws=None, status=None):
        torch, B = self.torch, len(self.lens)
        size = sp.sp_attend_tree_backward_workspace_bytes(self.dims, self.cache.desc, B)
        assert size > 0, sp.sp_last_error()
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") if ws is None else ws  # scratch holds NaN
        self.do_d = self.do.cuda()
        grads = grads or [torch.full_like(x, float("nan")) for x in self.rows]
        status = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
        torch.cuda.synchronize()
        sp.sp_attend_tree_backward(stream or torch.cuda.current_stream(), self.dims, self.cache.desc, B, None, self.lens_d,
                                   self.mask_d, self.n_d, *self.rows, self.out, self.lse, self.do_d, *grads, ws, size, status)
        torch.cuda.synchronize()
        self.status = int(status)
        return grads

    def reference(self, b):
        """Float64 gradients of sequence b and bounds of their errors; log sums and theirs."""
        torch, n, L = self.torch, self.N if self.n_nodes is None else self.n_nodes[b], self.lens[b]
        G, f32 = self.hq // self.hkv, self.dtype == sp.SP_F32
        K, V = (torch.cat([self.cache.values(b, L, c), x[b, :n].double()]) for c, x in (("k", self.k), ("v", self.v)))
        sees = torch.ones((n, L + n), dtype=torch.bool)
        for i in range(n):
            for j in range(n):
                sees[i, L + j] = bool((int(self.masks[b][i]) >> j) & 1)
        shapes = [(self.N, self.hq, self.dh), (self.N, self.hkv, self.dh), (self.N, self.hkv, self.dh)]
        want, lim = ([torch.zeros(s, dtype=torch.float64) for s in shapes] for _ in range(2))
        lse, lse_lim = (torch.zeros((n, self.hq), dtype=torch.float64) for _ in range(2))
        for h in range(self.hq if n else 0):
            k, v, q, do = K[:, h // G], V[:, h // G], self.q[b, :n, h].double(), self.do[b, :n, h].double()
            x = (q @ k.T * self.scale).masked_fill(~sees, -float("inf"))
            p = torch.softmax(x, -1).nan_to_num(0.0)
            dp, dpa = do @ v.T, do.abs() @ v.abs().T
            delta, delta_a = (p * dp).sum(-1, keepdim=True), (p * dpa).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            # a score is off by dh + 4 roundings of its sums (2^-22 each for the tensor cores' sums), the log
            # sum by as much and 2^-20 of its size
            score = (q.abs() @ k.abs().T * self.scale).amax(-1, keepdim=True) * (self.dh + 4) * (2.0 ** -22 if self.tensor else 2.0 ** -24)
            lse[:, h] = torch.logsumexp(x, -1)
            lse_lim[:, h] = score[:, 0] + 2.0 ** -16 + lse[:, h].abs().nan_to_num(0.0, 0.0) * 2.0 ** -20
            # weights move by both; sums of dh products; the rounded output in out.dout; ds (and p in dv of a
            # tensor product) rounded as an operand
            e = 2 * score + 2 * lse_lim[:, h:h + 1] + 2.0 ** -15 + (0 if f32 else 2.0 ** -8)
            op = 2.0 ** -8 if self.tensor else 0.0
            dse = p * (dpa + delta_a) * e + ds.abs() * op
            want[0][:n, h] = ds @ k * self.scale
            lim[0][:n, h] = (dse @ k.abs()) * self.scale
            want[1][:n, h // G] += ds[:, L:].T @ q * self.scale
            lim[1][:n, h // G] += dse[:, L:].T @ q.abs() * self.scale
            want[2][:n, h // G] += p[:, L:].T @ do
            lim[2][:n, h // G] += (p * (e + op))[:, L:].T @ do.abs()
        half = 2.0 ** -24 if f32 else 2.0 ** -8
        return want, [a + w.abs() * half * 1.01 + 1e-30 for a, w in zip(lim, want)], lse, lse_lim

    def check(self):
        torch = self.torch
        grads = self.forward().backward()
        assert self.status == 0
        for b in range(len(self.lens)):
            want, lim, lse, lse_lim = self.reference(b)
            n = len(lse)
            got = self.lse.view(len(self.lens), self.N, self.hq)[b].cpu().double()
            assert bool((got[n:] == -float("inf")).all())
            assert bool((((got[:n] - lse).abs() <= lse_lim) | (got[:n] == lse)).all())
            for name, g, w, m, x in zip("qkv", grads, want, lim, (self.q, self.k, self.v)):
                got = g.view(len(self.lens), self.N, -1)[b, :, :w[0].numel()].cpu().double().view(w.shape)
                assert bool(((got - w).abs() <= m).all()), (b, name, float(((got - w).abs() / m).max()))
                assert bool((got[n:] == 0).all())
        for g, x, s in zip(grads, self.rows, self.strides):
            if s:
                used = {id(self.rows[0]): self.hq}.get(id(x), self.hkv) * self.dh
                assert bool(g[:, used:].isnan().all())
        return grads


ALL = [(sp.SP_F32, sp.SP_F32), (sp.SP_BF16, sp.SP_BF16), (sp.SP_E4M3, sp.SP_BF16), (sp.SP_BF16, sp.SP_F32),
       (sp.SP_E4M3, sp.SP_F32), (sp.SP_F32, sp.SP_BF16)]


@pytest.mark.parametrize("cdt,dtype", ALL)
@pytest.mark.parametrize("page", [0, 16, 32, 64])
@pytest.mark.parametrize("dh,hq,hkv", [(128, 4, 2), (64, 3, 3), (32, 5, 1)])
def test_ragged_batches(torch, cdt, dtype, page, dh, hq, hkv):
    Case(torch, cdt, dtype, page, dh, hq, hkv, [0, 1, 15, 16, 63, 64, 65, 127, 128, 129, 200, 400], 5, seed=page + dh).check()


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
@pytest.mark.parametrize("G,N", [(1, 1), (4, 1), (5, 3), (4, 8), (3, 11), (4, 16), (1, 64), (5, 13), (4, 32), (5, 32), (4, 64),
                                 (8, 64), (40, 2)])
@pytest.mark.parametrize("page", [0, 16])
def test_rows_of_a_kv_head_from_one_to_many(torch, cdt, dtype, G, N, page):
    Case(torch, cdt, dtype, page, 128, 2 * G, 2, [0, 70, 300], N, seed=G * 64 + N).check()


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_trees_of_their_own_sizes_and_chains(torch, cdt, dtype):
    Case(torch, cdt, dtype, 16, 128, 8, 2, [100, 0, 33, 257, 50], 9, n_nodes=[9, 4, 0, 1, 8], seed=3).check()
    Case(torch, cdt, dtype, 0, 128, 4, 1, [50, 140, 3], 12, seed=5, chain=True).check()


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_gradients_as_parts_of_a_fused_one(torch, cdt, dtype):
    Case(torch, cdt, dtype, 16, 128, 4, 2, [80, 5], 6, seed=6, strides=(4 * 128 + 16, 2 * 128 + 8, 3 * 128)).check()


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_long_sequences_in_shares(torch, cdt, dtype):
    Case(torch, cdt, dtype, 16, 128, 4, 1, [5000, 17, 2600], 4, seed=7).check()
    Case(torch, cdt, dtype, 0, 128, 4, 1, [9001], 3, seed=8).check()


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
@pytest.mark.parametrize("scale,q_std", [(0.5, 1.0), (0.0, 6.0), (0.0, 0.01)])
def test_scales_and_sharp_rows(torch, cdt, dtype, scale, q_std):
    Case(torch, cdt, dtype, 16, 128, 4, 2, [300, 40], 5, seed=9, scale=scale, q_std=q_std).check()


@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("codes,least", [(256, 2.0 ** -10), (8, 8.0)])  # all; 0 and the subnormal ones
def test_every_code_of_an_8_bit_cache(torch, path, page, codes, least):
    c = Case(torch, sp.SP_E4M3, sp.SP_BF16, page, 128, 8, 2, [300, 130, 77], 5, path=path, seed=17)
    g = torch.Generator(device="cuda").manual_seed(17)
    for pool, scale in ((c.cache.k, c.cache.ks), (c.cache.v, c.cache.vs)):
        x = torch.randint(0, codes, pool.shape, generator=g, device="cuda", dtype=torch.int32)
        if codes == 8:
            x += 128 * torch.randint(0, 2, pool.shape, generator=g, device="cuda", dtype=torch.int32)
        pool.view(torch.uint8).copy_(torch.where((x & 127) == 127, 0, x).to(torch.uint8))
        scale.copy_(least * (1 + 7 * torch.rand(scale.shape, generator=g, device="cuda")))
    c.check()


@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("which", ["k", "v"])
def test_nan_codes_reach_their_sequence_alone(torch, path, which):
    lens = [70, 200]
    a = Case(torch, sp.SP_E4M3, sp.SP_BF16, 16, 128, 4, 2, lens, 3, path=path, seed=18)
    ga = a.forward().backward()
    b = Case(torch, sp.SP_E4M3, sp.SP_BF16, 16, 128, 4, 2, lens, 3, path=path, seed=18)
    b.forward()
    getattr(b.cache, which).view(torch.uint8)[b.cache._at(0, [50])[0], 0, b.cache._at(0, [50])[2], 3] = 0xff
    gb = b.backward()
    assert bool(gb[0][:3].view(3, 4, 128)[:, :2].isnan().any(-1).all())   # the heads of kv head 0
    assert torch.equal(gb[0][:3].view(3, 4, 128)[:, 2:], ga[0][:3].view(3, 4, 128)[:, 2:])
    assert torch.equal(gb[0][3:], ga[0][3:])
    for x, y in zip(ga[1:], gb[1:]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_log_sums_leave_the_output_as_it_is(torch, cdt, dtype):
    c = Case(torch, cdt, dtype, 16, 128, 8, 2, [100, 0, 333, 3000], 9, seed=10).forward()
    out, status = tree_call(torch, c.cache, c.dims, c.lens, c.mask_d, None, *c.rows)
    assert status == 0 and torch.equal(out.flatten(), c.out.cpu().flatten())


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_what_a_row_does_not_see_has_no_influence(torch, cdt, dtype):
    # node 2 is seen by itself alone; its key and value are NaN, and so is the cache past the ends
    lens, N = [70, 5], 4
    a = Case(torch, cdt, dtype, 16, 128, 4, 2, lens, N, seed=11)
    a.masks[:] = np.array([0b0001, 0b0011, 0b0100, 0b1011], np.uint64)
    ga = a.forward().backward()
    b = Case(torch, cdt, dtype, 16, 128, 4, 2, lens, N, seed=11)
    b.masks[:] = a.masks
    b.k[:, 2], b.v[:, 2] = float("nan"), float("inf")
    gb = b.forward().backward()
    others = [0, 1, 3, 4, 5, 7]
    for x, y in zip(ga, gb):
        assert torch.equal(x[others], y[others])
    assert bool(gb[0][[2, 6]].isnan().all())


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_rows_that_see_nothing(torch, cdt, dtype):
    c = Case(torch, cdt, dtype, 16, 128, 4, 2, [0, 0, 40], 3, n_nodes=[3, 0, 3], seed=12)
    c.masks[0][1] = 0  # an empty mask over an empty cache
    grads = c.check()
    assert bool((grads[0].view(3, 3, -1)[0, 1] == 0).all())


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_problems_are_reported(torch, cdt, dtype):
    c = Case(torch, cdt, dtype, 16, 128, 4, 2, [60, 60, 60], 3, seed=13).forward()
    c.lens_d[0], c.n_d = 1 << 20, torch.tensor([3, 7, 3], dtype=torch.int32).cuda()
    c.cache.table[2, 1] = 1 << 20
    c.cache.describe()
    c.cache.desc.max_seq_len = 60
    c.backward()
    assert c.status == sp.SP_DEV_BAD_LENGTH | sp.SP_DEV_BAD_PAGE | sp.SP_DEV_BAD_ROW


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_the_same_bits_every_time_captured_too(torch, cdt, dtype):
    c = Case(torch, cdt, dtype, 16, 128, 8, 2, [700, 3, 90, 2000], 7, seed=14).forward()
    want = c.backward()
    size = sp.sp_attend_tree_backward_workspace_bytes(c.dims, c.cache.desc, 4)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(x) for x in want]
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        sp.sp_attend_tree_backward(s, c.dims, c.cache.desc, 4, None, c.lens_d, c.mask_d, None, *c.rows, c.out, c.lse, c.do_d,
                                   *out, ws, size)
    for _ in range(2):
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_against_differences(torch):
    # the slope of sum(do o) along directions of q, k and v of the nodes, from the attention formula in
    # float64: h = 1e-4 leaves h^2 of third derivatives, the fp32 gradients 2^-13 of their terms' sum
    c = Case(torch, sp.SP_F32, sp.SP_F32, 16, 32, 4, 2, [20], 4, seed=15)
    dq, dk, dv = (x.cpu().double() for x in c.forward().backward())
    g = torch.Generator().manual_seed(16)
    u = [torch.randn(x[0].shape, generator=g).double() / 8 for x in (c.q, c.k, c.v)]
    K, V = c.cache.values(0, 20, "k"), c.cache.values(0, 20, "v")
    sees = torch.ones((4, 24), dtype=torch.bool)
    for i in range(4):
        for j in range(4):
            sees[i, 20 + j] = bool((int(c.masks[0][i]) >> j) & 1)

    def f(a):
        q, k, v = (x[0].double() + a * d for x, d in zip((c.q, c.k, c.v), u))
        k, v = torch.cat([K, k]), torch.cat([V, v])
        total = 0.0
        for h in range(4):
            x = (q[:, h] @ k[:, h // 2].T * 32 ** -0.5).masked_fill(~sees, -float("inf"))
            total += float((torch.softmax(x, -1) @ v[:, h // 2] * c.do[0, :, h].double()).sum())
        return total
    slope = (f(1e-4) - f(-1e-4)) / 2e-4
    parts = [x.view(d.shape) * d for x, d in zip((dq, dk, dv), u)]
    assert abs(slope - float(sum(p.sum() for p in parts))) <= float(sum(p.abs().sum() for p in parts)) * 2.0 ** -13 + 1e-6
