"""Decoding with drafted trees over a cache that a probe reads (one attention layer).

    python examples/tree_decode.py [--cache bf16|e4m3] [--batch 8] [--nodes 12] [--steps 6]

What a serving loop does with a draft model's tree, on the library's cache operators:

    prompts      keys rotated and written into the paged cache (quantised for e4m3) in one pass
    each step    queries and keys of the tree's nodes rotated in place inside the fused
                 projection's rows, every node attends to [cache ; its path], the accepted path
                 is appended to the cache
    at the end   contexts read back; with a bf16 cache the probe classifies the sequences from
                 the same pages, without another copy

Random rows stand in for the projections of a model's tokens, and a rule on the attention's
output for the verdict of the large model (which nodes it accepts).
"""
import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_28099_gb300 as sp  # noqa: E402


class TreeDecoder:
    """The cache of `batch` sequences and the calls of a decoding loop over it.

    A token's row is its fused projection, bf16 [(Hq + 2 Hkv) * dh]: queries, keys, values."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, max_len, max_nodes, cache_dtype=sp.SP_BF16,
                 page=16, theta=1.0e6, seed=0):
        import torch
        self.torch, self.B, self.N = torch, batch, max_nodes
        self.Hq, self.Hkv, self.dh, self.max_len = n_q_heads, n_kv_heads, head_dim, max_len
        self.width = (n_q_heads + 2 * n_kv_heads) * head_dim
        dev = "cuda"
        pages = -(-max_len // page)
        shape = (batch * pages, n_kv_heads, page, head_dim)
        kind = {sp.SP_BF16: torch.bfloat16, sp.SP_E4M3: torch.uint8}[cache_dtype]
        self.k_pool, self.v_pool = (torch.zeros(shape, dtype=kind, device=dev) for _ in range(2))
        scales = [None, None]
        if cache_dtype == sp.SP_E4M3:
            self.scales = [torch.zeros(shape[:3], device=dev) for _ in range(2)]
            scales = [s.data_ptr() for s in self.scales]
        order = np.random.default_rng(seed).permutation(batch * pages).astype(np.int32)
        self.table = torch.from_numpy(order.reshape(batch, pages)).to(dev)
        kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, self.k_pool.data_ptr(), self.v_pool.data_ptr(),
                            self.table.data_ptr(), page, batch * pages, pages, batch)
        self.cache = sp.sp_token_cache(kv, cache_dtype, n_kv_heads, head_dim, max_len, *scales)

        turns, amplitude = sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, head_dim, theta)
        self.turns = torch.from_numpy(turns.view(np.int64)).to(dev)
        self.rot = sp.sp_rotary(head_dim, head_dim, 0, amplitude, self.turns.data_ptr())
        self.dims = sp.sp_tree_dims(n_q_heads, max_nodes, sp.SP_BF16, 0, 0, 0.0, self.width, self.width, self.width)
        self.ws_bytes = sp.sp_attend_tree_workspace_bytes(self.dims, self.cache, batch)
        if self.ws_bytes == 0:
            raise sp.SpError(0, sp.sp_last_error())
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def _stream(self):
        return self.torch.cuda.current_stream()

    def _parts(self, rows):
        q, k = self.Hq * self.dh, self.Hkv * self.dh
        return rows[:, :q], rows[:, q:q + k], rows[:, q + k:]

    def _append(self, rows, row0, count, take, most, rot):
        _, k, v = self._parts(rows)
        where = sp.sp_token_rows(None if row0 is None else row0.data_ptr(), count.data_ptr(),
                                 None if take is None else take.data_ptr(), most, len(rows), self.width, self.width)
        sp.sp_cache_append(self._stream(), self.cache, rot, self.B, None, self.lens, where, sp.SP_BF16, k, v,
                           self.status)
        self.lens += count

    def prefill(self, rows, counts):
        """Prompts one behind another: rows of counts[b] tokens for sequence b, keys not yet rotated."""
        torch = self.torch
        row0 = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)[:-1]]).astype(np.int32)).cuda()
        self._append(rows, row0, torch.tensor(counts, dtype=torch.int32, device="cuda"), None, max(counts), self.rot)

    def attend(self, rows, parents):
        """rows [B * N][width] of the trees' nodes (rotated in place), parents: a list per sequence.
        The attention of every node, [B][N][Hq][dh]."""
        torch, B, N = self.torch, self.B, self.N
        masks, depths = np.zeros((B, N), np.uint64), np.zeros((B, N), np.int32)
        for b, tree in enumerate(parents):
            masks[b, :len(tree)], depths[b, :len(tree)] = sp.sp_tree_masks(tree)
        mask = torch.from_numpy(masks.view(np.int64)).cuda()
        n = torch.tensor([len(t) for t in parents], dtype=torch.int32, device="cuda")
        pos = (self.lens[:, None] + torch.from_numpy(depths).cuda()).flatten().contiguous()
        # queries and keys are neighbours in a row: one call turns both
        sp.sp_rotate(self._stream(), self.rot, B * N, pos, 0, sp.SP_BF16, self.Hq + self.Hkv, rows, self.width, self.dh,
                     rows, self.width, self.dh)
        q, k, v = self._parts(rows)
        out = torch.empty((B, N, self.Hq, self.dh), dtype=torch.bfloat16, device="cuda")
        sp.sp_attend_tree(self._stream(), self.dims, self.cache, B, None, self.lens, mask, n, q, k, v, out, self.ws,
                          self.ws_bytes, self.status)
        return out

    def accept(self, rows, paths):
        """The accepted nodes (a list per sequence, from the root on) join the cache."""
        torch = self.torch
        take = np.zeros((self.B, self.N), np.int32)
        for b, path in enumerate(paths):
            take[b, :len(path)] = path
        count = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
        self._append(rows, None, count, torch.from_numpy(take).cuda(), self.N, None)  # (rotated by attend)

    def read(self, dtype=sp.SP_F32):
        """Every sequence's keys and values, [B][longest][Hkv][dh] each (zeros past the ends)."""
        torch = self.torch
        most = int(self.lens.max())
        kind = torch.float32 if dtype == sp.SP_F32 else torch.bfloat16
        k, v = (torch.empty((self.B * most, self.Hkv, self.dh), dtype=kind, device="cuda") for _ in range(2))
        rows = sp.sp_token_rows(None, None, None, most, self.B * most, self.Hkv * self.dh, self.Hkv * self.dh)
        sp.sp_cache_read(self._stream(), self.cache, self.B, None, self.lens, None, rows, dtype, k, v, self.status)
        return (x.view(self.B, most, self.Hkv, self.dh) for x in (k, v))

    def check(self):
        bits = int(self.status.item())
        if bits:
            raise RuntimeError(f"device status {bits}")


def draft(rng, n):
    """A tree: chains that branch here and there."""
    return [int(rng.integers(-1, i)) if i and rng.random() < 0.4 else i - 1 for i in range(n)]


def path_to(tree, node):
    path = []
    while node >= 0:
        path.append(node)
        node = tree[node]
    return path[::-1]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--cache", choices=["bf16", "e4m3"], default="bf16")
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--nodes", type=int, default=12)
    ap.add_argument("--steps", type=int, default=6)
    a = ap.parse_args()
    import torch
    from paper_2608_28099_gb300 import build_lib
    from paper_2608_28099_gb300 import workloads as wl
    build_lib.build()
    rng = np.random.default_rng(1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    shape = wl.Shape(1024, 8, 2, 128, 2048, 4, 2)
    counts = [int(c) for c in rng.integers(40, 400, a.batch)]
    dec = TreeDecoder(a.batch, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, max(counts) + a.steps * a.nodes + 1,
                      a.nodes, {"bf16": sp.SP_BF16, "e4m3": sp.SP_E4M3}[a.cache], theta=shape.rope_theta)

    def rows(n):
        return torch.randn((n, dec.width), generator=gen, device="cuda").to(torch.bfloat16)

    dec.prefill(rows(sum(counts)), counts)
    for step in range(a.steps):
        trees = [draft(rng, int(rng.integers(1, a.nodes + 1))) for _ in range(a.batch)]
        nodes = rows(a.batch * a.nodes)
        out = dec.attend(nodes, trees)
        score = out.float().mean((2, 3)).cpu().numpy()  # stands in for the large model's verdict
        paths = [path_to(t, int(np.argmax(score[b, :len(t)]))) for b, t in enumerate(trees)]
        dec.accept(nodes, paths)
        print(f"step {step}: {sum(map(len, trees))} nodes drafted, {sum(map(len, paths))} accepted, "
              f"lengths {dec.lens.tolist()}")
    k, v = dec.read()
    dec.check()
    print(f"contexts read back: {tuple(k.shape)}, largest key {k.abs().max().item():.3f}, value {v.abs().max().item():.3f}")
    if a.cache == "bf16":
        weights = wl.draw_weights(shape, np.random.default_rng(2), False)
        model = sp.Model(shape, weights, a.batch, dec.max_len)
        ids = torch.arange(a.batch, dtype=torch.int32, device="cuda")
        logits = torch.empty((a.batch, shape.n_classes), device="cuda")
        sp.sp_classify(model.handle, torch.cuda.current_stream(), a.batch, ids, dec.lens, dec.cache.kv, None, logits)
        bits = sp.sp_check_status(model.handle)
        if bits:
            raise RuntimeError(f"device status {bits}: {sp.sp_last_error()}")
        print("probe's classes:", logits.argmax(1).tolist())
        model.close()


if __name__ == "__main__":
    main()
