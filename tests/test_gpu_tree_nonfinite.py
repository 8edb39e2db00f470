"""NaN and infinities that a row sees reach it on every path of the tree attention,
wherever they lie among the tiles, copies, pipelines and shares of a call."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_tree import tree_call
from token_cache_util import Cache, mask_tensor

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
KINDS = [(sp.SP_BF16, 1), (sp.SP_BF16, 2), (sp.SP_E4M3, 1), (sp.SP_E4M3, 2)]
ROWS = [(1, 4), (4, 13), (4, 25), (4, 50)]  # query heads a kv head, nodes: 4, 52, 100, 200 rows
HKV, DH = 2, 128


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


class Call:
    """A batch of chains over a cache whose tensors a test changes between runs."""

    def __init__(self, torch, cdt, path, G, N, lens, page=16, seed=0, scale=0.0, mask=None):
        self.torch, self.G, self.N, self.lens = torch, G, N, lens
        g = torch.Generator().manual_seed(seed + 31 * N)
        self.cache = Cache(cdt, HKV, DH, [max(x, 1) for x in lens], page, seed)
        self.kv = [[torch.randn((n, HKV, DH), generator=g) for _ in range(2)] for n in lens]
        B = len(lens)
        self.q, self.k, self.v = (torch.randn((B, N, h, DH), generator=g).to(torch.bfloat16) for h in (G * HKV, HKV, HKV))
        self.dims = sp.sp_tree_dims(G * HKV, N, sp.SP_BF16, path, 0, scale, 0, 0, 0)
        self.mask = None if mask is None else mask_tensor(torch, np.stack([np.array(mask, np.uint64)] * B))

    def run(self):
        for s, (k, v) in enumerate(self.kv):
            if len(k):
                self.cache.put(s, 0, k, v)
        out, status = tree_call(self.torch, self.cache, self.dims, self.lens, self.mask, None, self.q.cuda(),
                                self.k.cuda(), self.v.cuda())
        assert status == 0
        return out

    def heads(self, g):
        return slice(g * self.G, (g + 1) * self.G)


def same_elsewhere(torch, got, clean, touched):
    assert bool(torch.isfinite(clean).all())
    assert torch.equal(got[~touched], clean[~touched])


def check_query(torch, cdt, path, G, N, lens, value):
    c = Call(torch, cdt, path, G, N, lens)
    clean = c.run()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    for b in range(len(lens)):
        for i, h in ((0, 0), (N - 1, 2 * G - 1), (N // 2, G - 1)):
            c.q[b, i, h, 17 * b % DH] = value
            touched[b, i, h] = True
    got = c.run()
    assert bool(torch.isnan(got[touched]).all())
    same_elsewhere(torch, got, clean, touched)


def check_cached_key(torch, cdt, path, G, N, length, tokens):
    c = Call(torch, cdt, path, G, N, [length, 20, length])
    clean = c.run()
    c.kv[0][0][tokens, 0, 3] = NAN
    c.kv[2][0][tokens, 1, 127] = NAN
    got = c.run()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[0, :, c.heads(0)] = touched[2, :, c.heads(1)] = True
    assert bool(torch.isnan(got[touched]).all())
    same_elsewhere(torch, got, clean, touched)


# ---- one share a sequence: two tiles at most --------------------------------
@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
def test_a_nan_query(torch, cdt, path, G, N):
    check_query(torch, cdt, path, G, N, [0, 1, 33, 100, 128], NAN)


@pytest.mark.parametrize("G,N", ROWS)
def test_an_infinite_query_over_an_8_bit_cache(torch, G, N):
    check_query(torch, sp.SP_E4M3, 2, G, N, [1, 33, 100, 128], INF)


@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("length", [1, 33, 65, 97, 128])
def test_a_nan_key_alone_in_its_copy_or_tile(torch, cdt, path, G, N, length):
    check_cached_key(torch, cdt, path, G, N, length, [length - 1])


@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
def test_a_nan_key_of_a_node(torch, cdt, path, G, N):
    # node 0 hangs alone on an empty or a short cache; the last node is seen by itself only;
    # the others see neither
    masks = [1] + [1 << i | (2 if i > 1 else 0) for i in range(1, N)]
    c = Call(torch, cdt, path, G, N, [0, 40, 0], mask=masks)
    clean = c.run()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    for i in (0, N - 1):
        c.k[:, i, 1, 5] = NAN
        touched[:, i, c.heads(1)] = True
    got = c.run()
    assert bool(torch.isnan(got[touched]).all())
    same_elsewhere(torch, got, clean, touched)


# ---- sequences that are cut ---------------------------------------------------
@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
def test_a_nan_query_of_a_split_sequence(torch, cdt, path, G, N):
    check_query(torch, cdt, path, G, N, [3000, 129, 700], NAN)


@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("tokens", [[0], [2999], list(range(1500))], ids=["first", "last", "half"])
def test_nan_keys_of_a_split_sequence(torch, cdt, path, G, N, tokens):
    check_cached_key(torch, cdt, path, G, N, 3000, tokens)


@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
def test_a_nan_key_alone_in_a_pipeline(torch, cdt, path, G, N):
    check_cached_key(torch, cdt, path, G, N, 129, [128])


# ---- scales --------------------------------------------------------------------
@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("which", ["ks", "vs"])
@pytest.mark.parametrize("G,N", ROWS)
def test_a_nan_scale(torch, path, page, which, G, N):
    # the token's values, or its score, are NaN; the next call finds what this one left in
    # shared memory and must not be touched by it
    c = Call(torch, sp.SP_E4M3, path, G, N, [40, 300, 7], page)
    clean = c.run()
    c.run()
    scales = getattr(c.cache, which)
    for s, t in ((0, 39), (1, 5)):
        at = c.cache._at(s, [t])
        row = scales[at].clone()
        row[..., 0] = NAN
        scales[at] = row
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[:2, :, c.heads(0)] = True

    def call():
        out, status = tree_call(torch, c.cache, c.dims, c.lens, None, None, c.q.cuda(), c.k.cuda(), c.v.cuda())
        assert status == 0
        return out
    got = call()
    assert bool(torch.isnan(got[touched]).all())
    same_elsewhere(torch, got, clean, touched)
    assert torch.equal(c.run(), clean)
