"""Token caches for the tests of the cache operators: built on the host in float64
values, laid out as the library takes them, and the attention of a tree over them in
float64 from its definition."""
from __future__ import annotations

import numpy as np

import paper_2608_28099_gb300 as sp

ES = {sp.SP_F32: 4, sp.SP_BF16: 2, sp.SP_E4M3: 1}


def torch_type(dtype):
    import torch
    return {sp.SP_F32: torch.float32, sp.SP_BF16: torch.bfloat16, sp.SP_E4M3: torch.float8_e4m3fn}[dtype]


def quantise(x):
    """(codes as float8, scales) of fp32 rows by the documented formula."""
    import torch
    finite = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    amax = finite.amax(-1).clamp_min(2.0 ** -60)
    y = x * (torch.full_like(amax, 448.0) / amax)[..., None]  # (a scalar over a tensor is not one division)
    y = torch.where(torch.isfinite(x), y, torch.full_like(y, float("nan")))
    return y.to(torch.float8_e4m3fn), amax / 448.0


class Cache:
    """A cache of n_seqs sequences on the GPU.  room[s]: tokens sequence s can hold;
    page 0 = contiguous.  Every element starts as `junk` (also past the ends)."""

    def __init__(self, dtype, hkv, dh, room, page, seed=0, junk=float("nan"), spare_pages=3):
        import torch
        self.torch, self.dtype, self.hkv, self.dh, self.page, self.room = torch, dtype, hkv, dh, page, list(room)
        rng = np.random.default_rng(seed)
        self.max_len = max(max(room), 1)
        n = len(room)
        t = torch_type(dtype)
        if page:
            pages = [-(-r // page) for r in room]
            self.n_pages = sum(pages) + spare_pages
            perm = rng.permutation(self.n_pages)
            self.table = np.full((n, max(max(pages), 1)), -1, np.int32)
            at = 0
            for s, p in enumerate(pages):
                self.table[s, :p] = perm[at:at + p]
                at += p
            shape, sshape = (self.n_pages, hkv, page, dh), (self.n_pages, hkv, page)
        else:
            self.start = np.concatenate([[0], np.cumsum(room)]).astype(np.int64)
            shape, sshape = (int(self.start[-1]) + 1, hkv, dh), (int(self.start[-1]) + 1, hkv)
        self.k = torch.full(shape, junk).to(t).cuda()
        self.v = torch.full(shape, junk).to(t).cuda()
        self.ks = self.vs = None
        if dtype == sp.SP_E4M3:
            self.ks, self.vs = (torch.full(sshape, 1.0).cuda() for _ in range(2))
        self.describe()

    def describe(self):
        torch, n = self.torch, len(self.room)
        if self.page:
            self.table_d = torch.from_numpy(self.table).cuda()
            kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, self.k.data_ptr(), self.v.data_ptr(),
                                self.table_d.data_ptr(), self.page, self.n_pages, self.table.shape[1], n)
            sc = [None if t is None else t.data_ptr() for t in (self.ks, self.vs)]
        else:
            row = self.hkv * self.dh * ES[self.dtype]
            self.ptrs = [torch.from_numpy(t.data_ptr() + self.start[:-1] * row).cuda() for t in (self.k, self.v)]
            kv = sp.sp_kv_cache(sp.SP_KV_CONTIGUOUS, self.ptrs[0].data_ptr(), self.ptrs[1].data_ptr(), None, None,
                                None, 0, 0, 0, n)
            sc = [None, None]
            if self.ks is not None:
                self.ptrs += [torch.from_numpy(t.data_ptr() + self.start[:-1] * (self.hkv * 4)).cuda()
                              for t in (self.ks, self.vs)]
                sc = [t.data_ptr() for t in self.ptrs[2:]]
        self.desc = sp.sp_token_cache(kv, self.dtype, self.hkv, self.dh, self.max_len, *sc)

    def _at(self, s, tokens):
        tokens = np.asarray(tokens, np.int64)
        if self.page:
            pages = self.torch.from_numpy(self.table[s].astype(np.int64))[tokens // self.page].cuda()
            return pages, slice(None), self.torch.from_numpy(tokens % self.page).cuda()
        return (self.torch.from_numpy(self.start[s] + tokens).cuda(),)

    def put(self, s, first, k, v):
        """Write fp32 rows [n][hkv][dh] (quantised by the formula) from token `first` on."""
        at = self._at(s, np.arange(first, first + len(k)))
        for pool, scale, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            x = x.cuda()
            if scale is not None:
                q, sc = quantise(x)
                pool.view(self.torch.uint8)[at] = q.view(self.torch.uint8)
                scale[at] = sc
            else:
                pool[at] = x.to(pool.dtype)

    def values(self, s, n, which):
        """float64 values [n][hkv][dh] of the first n tokens."""
        pool, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        at = self._at(s, np.arange(n))
        raw = pool.view(self.torch.uint8)[at].view(pool.dtype) if scale is not None else pool[at]
        x = raw.float().double()
        return (x if scale is None else x * scale[at].double()[..., None]).cpu()

    def codes(self, s, n, which):
        pool = self.k if which == "k" else self.v
        at = self._at(s, np.arange(n))
        x = pool.view({4: self.torch.int32, 2: self.torch.int16, 1: self.torch.uint8}[pool.element_size()])
        return x[at].cpu()

    def scales(self, s, n, which):
        return (self.ks if which == "k" else self.vs)[self._at(s, np.arange(n))].cpu()


def random_parents(rng, n):
    return [int(rng.integers(-1, i)) if i and rng.random() < 0.5 else i - 1 for i in range(n)]


def mask_tensor(torch, masks):
    return torch.from_numpy(np.ascontiguousarray(masks, np.uint64).view(np.int64)).cuda()


def tree_reference(cache, s, L, q, k_new, v_new, mask, scale):
    """Float64 attention of nodes q [n][Hq][dh] of sequence s over its L cached tokens
    and its nodes; mask [n] ints.  Returns (o, the same with |v| for v, the largest
    sum |q k| scale of a row): the last two scale the error bounds."""
    import torch
    n, hq, dh = q.shape
    hkv = cache.hkv
    G = hq // hkv
    K = torch.cat([cache.values(s, L, "k"), k_new.double()])
    V = torch.cat([cache.values(s, L, "v"), v_new.double()])
    sees = torch.ones((n, L + n), dtype=torch.bool)
    for i in range(n):
        for j in range(n):
            sees[i, L + j] = bool((int(mask[i]) >> j) & 1)
    o, oa = torch.zeros((n, hq, dh), dtype=torch.float64), torch.zeros((n, hq, dh), dtype=torch.float64)
    spread = 0.0
    for h in range(hq):
        for i in range(n):
            vis = sees[i]
            if not bool(vis.any()):
                continue
            k, v = K[vis, h // G], V[vis, h // G]
            x = (k @ q[i, h].double()) * scale
            spread = max(spread, float((k.abs() @ q[i, h].double().abs()).max()) * scale)
            p = torch.softmax(x, 0)
            o[i, h] = p @ v
            oa[i, h] = p @ v.abs()
    return o, oa, spread
