"""Attention of drafted trees over [cache ; tree] against float64, on every path."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from token_cache_util import Cache, mask_tensor, random_parents, torch_type, tree_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def tree_call(torch, cache, dims, lens, mask, n_nodes, q, k, v, ids=None, max_len=None, stream=None, batch=None):
    B = batch or len(lens)
    if max_len is not None:
        cache.desc.max_seq_len = max_len
    size = sp.sp_attend_tree_workspace_bytes(dims, cache.desc, B)
    assert size > 0, sp.sp_last_error()
    ws = torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda")  # scratch holds anything
    out = torch.full((B * dims.n_nodes, dims.n_q_heads, cache.dh), float("nan")).to(torch_type(dims.dtype)).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    sp.sp_attend_tree(stream or torch.cuda.current_stream(), dims, cache.desc, B, ids,
                      torch.tensor(lens, dtype=torch.int32).cuda(), mask,
                      None if n_nodes is None else torch.tensor(n_nodes, dtype=torch.int32).cuda(), q, k, v, out, ws, size,
                      status)
    torch.cuda.synchronize()
    return out.view(B, dims.n_nodes, dims.n_q_heads, cache.dh).cpu(), int(status.item())


def bound(o, oa, spread, dtype, cdt, tensor, dh=128):
    """Largest error of the arithmetic.  A score is off by (dh + 4) roundings of its
    partial sums (fp32; 2^-22 each for the tensor cores' sums; 2^-17 in all for queries
    split into 8-bit parts), which moves the weights by twice that; fp32 weights and
    sums add 2^-18 of sum p |v|, bf16 weights (8 bits: 2^-8 of each) 2^-7 with their
    sum's, 16-bit float weights (11 bits) and values 2^-10; a bf16 result 2^-8 of itself."""
    score = spread * (dh + 4) * (2.0 ** -22 if tensor else 2.0 ** -24)
    if tensor and cdt == sp.SP_E4M3:
        score += spread * 2.0 ** -17
    weight = 2.0 ** -18 if not tensor else 2.0 ** -7 if cdt == sp.SP_BF16 else 2.0 ** -10
    out = 2.0 ** -8 if dtype == sp.SP_BF16 else 2.0 ** -23
    return oa * (2 * score + weight) + out * o.abs() * 1.01 + 1e-30


def fill(torch, cache, lens, seed, k_std=1.0):
    g = torch.Generator().manual_seed(seed)
    for s, n in enumerate(lens):
        k, v = (torch.randn((n, cache.hkv, cache.dh), generator=g) for _ in range(2))
        cache.put(s, 0, k * k_std, v * torch.exp(torch.randn((n, cache.hkv, 1), generator=g)))
    return g


def check(torch, cdt, dtype, page, dh, hq, hkv, lens, N, n_nodes=None, path=0, seed=0, tensor=None, scale=0.0,
          shared=False, chain=False, q_std=1.0):
    cache = Cache(cdt, hkv, dh, [max(x, 1) for x in lens], page, seed)
    g = fill(torch, cache, lens, seed)
    rng = np.random.default_rng(seed)
    B, t = len(lens), torch_type(dtype)
    q = (torch.randn((B, N, hq, dh), generator=g) * q_std).to(t)
    k, v = (torch.randn((B, N, hkv, dh), generator=g).to(t) for _ in range(2))
    masks = np.stack([sp.sp_tree_masks(random_parents(rng, N))[0] for _ in range(1 if shared else B)])
    if chain:
        masks = np.stack([sp.sp_tree_masks(list(range(-1, N - 1)))[0]])
    dims = sp.sp_tree_dims(hq, N, dtype, path, int(shared), scale, 0, 0, 0)
    out, status = tree_call(torch, cache, dims, lens, None if chain else mask_tensor(torch, masks), n_nodes, q.cuda(),
                            k.cuda(), v.cuda())
    assert status == 0
    if tensor is None:
        tensor = dtype == sp.SP_BF16 and dh == 128 and cdt != sp.SP_F32 and path != 1
    worst = 0.0
    for b in range(B):
        n = N if n_nodes is None else n_nodes[b]
        o, oa, spread = tree_reference(cache, b, lens[b], q[b, :n], k[b, :n], v[b, :n],
                                       masks[b if len(masks) > 1 else 0], scale or dh ** -0.5)
        err = (out[b, :n].double() - o).abs()
        lim = bound(o, oa, spread, dtype, cdt, tensor, dh)
        assert bool((err <= lim).all()), (b, float((err / lim).max()))
        worst = max(worst, float((err / lim).max()) if n else 0.0)
        assert bool((out[b, n:] == 0).all())
    return worst


ALL = [(sp.SP_F32, sp.SP_F32), (sp.SP_BF16, sp.SP_BF16), (sp.SP_E4M3, sp.SP_BF16), (sp.SP_BF16, sp.SP_F32),
       (sp.SP_E4M3, sp.SP_F32), (sp.SP_F32, sp.SP_BF16)]


@pytest.mark.parametrize("cdt,dtype", ALL)
@pytest.mark.parametrize("page", [0, 16, 32, 64])
@pytest.mark.parametrize("dh,hq,hkv", [(128, 4, 2), (64, 3, 3), (32, 5, 1)])
def test_ragged_batches(torch, cdt, dtype, page, dh, hq, hkv):
    check(torch, cdt, dtype, page, dh, hq, hkv, [0, 1, 15, 16, 63, 64, 127, 128, 129, 200, 400], 5, seed=page + dh)


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("G,N", [(1, 1), (4, 1), (5, 3), (4, 8), (3, 11), (4, 13), (4, 16), (1, 64), (5, 13), (4, 32),
                                 (5, 32), (4, 64), (5, 64), (8, 64)])
@pytest.mark.parametrize("page", [0, 16])
def test_rows_of_a_kv_head_from_one_to_many(torch, cdt, G, N, page):
    # the row counts that the kernels cut into tiles, copies and blocks: 1 .. 512
    check(torch, cdt, sp.SP_BF16, page, 128, 2 * G, 2, [0, 70, 300], N, seed=G * 64 + N)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_trees_of_their_own_sizes(torch, cdt, dtype):
    check(torch, cdt, dtype, 16, 128, 8, 2, [100, 0, 33, 257, 50], 9, n_nodes=[9, 4, 0, 1, 8], seed=3)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_one_tree_for_the_batch_and_a_chain(torch, cdt, dtype):
    check(torch, cdt, dtype, 16, 128, 4, 1, [50, 140, 3], 12, seed=4, shared=True)
    check(torch, cdt, dtype, 0, 128, 4, 1, [50, 140, 3], 12, seed=5, chain=True)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
@pytest.mark.parametrize("path", [0, 1])
def test_long_sequences_split_over_many_shares(torch, cdt, dtype, path):
    check(torch, cdt, dtype, 32, 128, 4, 2, [5000, 37, 2500], 6, seed=6, path=path)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_scores_that_keep_growing(torch, cdt, dtype):
    # large scores: the running maximum moves often, weights span all of fp32's range
    check(torch, cdt, dtype, 16, 128, 4, 2, [700, 300], 7, seed=7, q_std=25.0)
    check(torch, cdt, dtype, 16, 128, 4, 2, [700, 300], 7, seed=8, scale=2.5)
    check(torch, cdt, dtype, 16, 128, 4, 2, [700, 300], 7, seed=9, q_std=1e-6)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_rows_that_see_nothing_give_zeros(torch, cdt, dtype):
    N, hq, hkv, dh = 6, 4, 2, 128
    cache = Cache(cdt, hkv, dh, [20, 20], 16)
    g = fill(torch, cache, [0, 20], 1)
    t = torch_type(dtype)
    q, k, v = (torch.randn((2, N, h, dh), generator=g).to(t).cuda() for h in (hq, hkv, hkv))
    masks = np.array([[0, 2, 0, 1 << 5, 0, 63], [0, 0, 0, 0, 0, 0]], np.uint64)
    dims = sp.sp_tree_dims(hq, N, dtype, 0, 0, 0.0, 0, 0, 0)
    out, status = tree_call(torch, cache, dims, [0, 20], mask_tensor(torch, masks), None, q, k, v)
    assert status == 0 and bool((out[0, [0, 2, 4]] == 0).all())
    for i, j in ((1, 1), (3, 5)):  # one visible key: its value
        want = v[0, j].cpu().double().repeat_interleave(hq // hkv, 0)
        assert bool(((out[0, i].double() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-6).all())
    # (bf16: one weight of 1, exact; 8-bit caches: the value is a 16-bit float, exact)
    o, oa, spread = tree_reference(cache, 1, 20, q[1].cpu(), k[1].cpu(), v[1].cpu(), masks[1], dh ** -0.5)
    assert bool(((out[1].double() - o).abs() <= bound(o, oa, spread, dtype, cdt, dtype == sp.SP_BF16)).all())


@pytest.mark.parametrize("cdt,dtype", ALL)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_what_a_row_does_not_see_has_no_influence(torch, cdt, dtype, page, junk):
    N, hq, hkv, dh = 8, 4, 2, 128
    lens = [37, 130, 0]
    cache = Cache(cdt, hkv, dh, [x + 20 for x in lens], page, junk=float("nan"))
    g = fill(torch, cache, lens, 2)
    t = torch_type(dtype)
    q, k, v = (torch.randn((3, N, h, dh), generator=g).to(t).cuda() for h in (hq, hkv, hkv))
    masks = np.stack([sp.sp_tree_masks([-1, 0, 0, 1, 2, 0, -1, 6])[0]] * 3)
    dims = sp.sp_tree_dims(hq, N, dtype, 0, 0, 0.0, 0, 0, 0)
    n_nodes = [8, 8, 6]
    clean, _ = tree_call(torch, cache, dims, lens, mask_tensor(torch, masks), n_nodes, q, k, v)
    k[:, 4], v[:, 4, 1, 3] = junk, junk      # node 4, seen by itself only
    v[:, 6, 0, 7] = -junk                    # node 6, seen by 6 and 7
    k[2, 6:], v[2, 6:], q[2, 6:] = junk, junk, junk  # past the third tree's end
    out, status = tree_call(torch, cache, dims, lens, mask_tensor(torch, masks), n_nodes, q, k, v)
    assert status == 0
    for b in range(3):
        keep = [i for i in range(n_nodes[b]) if i not in (4, 6, 7)]
        assert torch.equal(out[b, keep], clean[b, keep])
        assert bool((out[b, n_nodes[b]:] == 0).all())
        assert not bool(torch.isfinite(out[b, 4]).any())
    for b in range(2):  # a value's own dim, and only it
        for i in (6, 7):
            bad = ~torch.isfinite(out[b, i])
            assert bool(bad[:2, 7].all()) and int(bad.sum()) == 2
            rest = ~bad
            assert torch.equal(out[b, i][rest], clean[b, i][rest])


@pytest.mark.parametrize("path", [0, 1])
def test_strided_rows_of_a_fused_projection(torch, path):
    hq, hkv, dh, N, lens = 4, 2, 128, 5, [90, 17]
    width = (hq + 2 * hkv) * dh + 64
    cache = Cache(sp.SP_E4M3, hkv, dh, lens, 16)
    g = fill(torch, cache, lens, 3)
    buf = torch.randn((2 * N, width), generator=g).to(torch.bfloat16).cuda()
    masks = mask_tensor(torch, np.stack([sp.sp_tree_masks([-1, 0, 0, 1, 1])[0]] * 2))
    q, k, v = (buf[:, a * dh:b * dh].contiguous() for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    dense, _ = tree_call(torch, cache, sp.sp_tree_dims(hq, N, sp.SP_BF16, path, 0, 0.0, 0, 0, 0), lens, masks, None, q, k, v)
    p = buf.data_ptr()
    strided, _ = tree_call(torch, cache, sp.sp_tree_dims(hq, N, sp.SP_BF16, path, 0, 0.0, width, width, width), lens, masks,
                           None, p, p + 2 * hq * dh, p + 2 * (hq + hkv) * dh)
    assert torch.equal(dense, strided)


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_results_repeat_bit_for_bit_on_any_stream_and_leave_the_cache_alone(torch, cdt, dtype):
    hq, hkv, dh, N, lens = 8, 2, 128, 12, [1500, 3, 700, 0, 260]
    cache = Cache(cdt, hkv, dh, [max(x, 1) for x in lens], 16)
    g = fill(torch, cache, lens, 4)
    t = torch_type(dtype)
    q, k, v = (torch.randn((5, N, h, dh), generator=g).to(t).cuda() for h in (hq, hkv, hkv))
    masks = mask_tensor(torch, np.stack([sp.sp_tree_masks(random_parents(np.random.default_rng(i), N))[0] for i in range(5)]))
    dims = sp.sp_tree_dims(hq, N, dtype, 0, 0, 0.0, 0, 0, 0)
    pools = [x.clone() for x in (cache.k, cache.v)]
    first, _ = tree_call(torch, cache, dims, lens, masks, None, q, k, v)
    side = torch.cuda.Stream()
    for _ in range(3):
        again, _ = tree_call(torch, cache, dims, lens, masks, None, q, k, v, stream=side)
        assert torch.equal(first, again)
    for a, b in zip(pools, (cache.k, cache.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("cdt,dtype", ALL[:3])
def test_ids_choose_sequences_and_bad_ones_are_reported(torch, cdt, dtype):
    hq, hkv, dh, N, lens = 4, 2, 128, 3, [40, 300, 7]
    cache = Cache(cdt, hkv, dh, lens, 16)
    g = fill(torch, cache, lens, 5)
    t = torch_type(dtype)
    q, k, v = (torch.randn((2, N, h, dh), generator=g).to(t).cuda() for h in (hq, hkv, hkv))
    dims = sp.sp_tree_dims(hq, N, dtype, 0, 0, 0.0, 0, 0, 0)
    tensor = dtype == sp.SP_BF16

    def run(ids, **kw):
        return tree_call(torch, cache, dims, kw.pop("lens", lens), None, None, q, k, v,
                         ids=torch.tensor(ids, dtype=torch.int32).cuda(), batch=2, **kw)
    out, status = run([2, 1])
    assert status == 0
    chain = sp.sp_tree_masks([-1, 0, 1])[0]
    for b, s in enumerate([2, 1]):
        o, oa, spread = tree_reference(cache, s, lens[s], q[b].cpu(), k[b].cpu(), v[b].cpu(), chain, dh ** -0.5)
        assert bool(((out[b].double() - o).abs() <= bound(o, oa, spread, dtype, cdt, tensor)).all())
    assert run([0, 3])[1] == sp.SP_DEV_BAD_SEQ_ID
    assert run([0, -1])[1] == sp.SP_DEV_BAD_SEQ_ID
    assert run([0, 1], lens=[40, 301, 7])[1] == sp.SP_DEV_BAD_LENGTH
    cache.table[1, 2] = cache.n_pages
    cache.table[0, 2] = -1
    cache.describe()
    out2, status = run([2, 1])
    assert status == sp.SP_DEV_BAD_PAGE and torch.equal(out2[0], out[0])
    assert run([0, 2])[1] == sp.SP_DEV_BAD_PAGE


def test_offsets_past_32_bits(torch):
    """A pool of more than 2^31 elements: the sequence's pages sit at both ends."""
    hkv, dh, P, N, hq = 8, 128, 64, 4, 8
    n_pages = 2 ** 32 // (hkv * dh * P) + 40
    L = 3 * P + 5
    small = Cache(sp.SP_E4M3, hkv, dh, [L], P, spare_pages=0)
    g = fill(torch, small, [L], 6)
    q, k, v = (torch.randn((1, N, h, dh), generator=g).to(torch.bfloat16).cuda() for h in (hq, hkv, hkv))
    dims = sp.sp_tree_dims(hq, N, sp.SP_BF16, 0, 0, 0.0, 0, 0, 0)
    want, _ = tree_call(torch, small, dims, [L], None, None, q, k, v)
    at = [n_pages - 1, 0, n_pages - 17, n_pages // 2]
    old = torch.from_numpy(small.table[0].astype(np.int64)).cuda()
    big = {}
    for name in ("k", "v", "ks", "vs"):
        src = getattr(small, name)
        dst = torch.zeros((n_pages,) + tuple(src.shape[1:]), dtype=torch.uint8 if name in "kv" else torch.float32, device="cuda")
        dst[torch.tensor(at).cuda()] = (src.view(torch.uint8) if name in "kv" else src)[old]
        big[name] = dst.view(torch.float8_e4m3fn) if name in "kv" else dst
    for name, t in big.items():
        setattr(small, name, t)
    small.table, small.n_pages = np.array([at], np.int32), n_pages
    small.describe()
    for path in (0, 1):
        dims.path = path
        got, status = tree_call(torch, small, dims, [L], None, None, q, k, v)
        assert status == 0
        if path == 0:
            assert torch.equal(got, want)
        else:  # bf16 of the same value within the two paths' bounds
            assert bool(((got.double() - want.double()).abs() <= 2.0 ** -6 * want.double().abs() + 2.0 ** -8).all())


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("N,page", [(4, 16), (13, 0), (16, 16), (25, 32), (40, 16)])
def test_long_shares_of_many_sequences(torch, cdt, N, page):
    # dozens of tiles and several sequences a block: rings wrap, segments follow one
    # another; every launch gives the same bits, near the fp32 kernel's result
    hkv, hq, dh, B = 8, 32, 128, 48
    rng = np.random.default_rng(N)
    lens = [int(x) for x in rng.integers(0, 3000, B)]
    cache = Cache(cdt, hkv, dh, [max(x, 1) for x in lens], page, junk=0.0)
    g = torch.Generator(device="cuda").manual_seed(N)
    for pool in (cache.k, cache.v):
        pool.copy_(torch.randn(pool.shape, generator=g, device="cuda").mul_(1 if cdt == sp.SP_BF16 else 60).to(pool.dtype))
    if cdt == sp.SP_E4M3:
        for sc in (cache.ks, cache.vs):
            sc.copy_(torch.rand(sc.shape, generator=g, device="cuda") / 40)
    q, k, v = (torch.randn((B, N, h, dh), generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    masks = mask_tensor(torch, np.stack([sp.sp_tree_masks(random_parents(rng, N))[0] for _ in range(B)]))
    n_nodes = [int(x) for x in rng.integers(0, N + 1, B)]
    dims = sp.sp_tree_dims(hq, N, sp.SP_BF16, 2, 0, 0.0, 0, 0, 0)
    first, status = tree_call(torch, cache, dims, lens, masks, n_nodes, q, k, v)
    assert status == 0
    args = [torch.tensor(x, dtype=torch.int32).cuda() for x in (lens, n_nodes)]
    size = sp.sp_attend_tree_workspace_bytes(dims, cache.desc, B)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    outs = [torch.empty((B, N, hq, dh), dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(400):
        sp.sp_attend_tree(stream, dims, cache.desc, B, None, args[0], masks, args[1], q, k, v, outs[i % 8], ws, size)
    torch.cuda.synchronize()
    assert all(torch.equal(o.cpu(), first) for o in outs)
    dims.path = 1
    ref, _ = tree_call(torch, cache, dims, lens, masks, n_nodes, q, k, v)
    # two bf16 roundings of the result, weights of 8 bits: 2^-8 each, in the 2-norm
    assert float((first.double() - ref.double()).norm()) <= 3 * 2.0 ** -8 * float(ref.double().norm())
