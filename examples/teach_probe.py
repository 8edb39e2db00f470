"""Teaching a probe: a soft prompt's gradient through the frozen draft layer (one layer).

    python examples/teach_probe.py [--batch 16] [--rows 8] [--steps 20] [--vocab 2000]

The layer and the head stay as they are; the soft prompt's rows, shared by all sequences, are
taught to make the head's token after them a given one (a label word).  Forward and backward run on the
library's calls; the projections' backward passes are products with the transposed weights,
laid out once:

    norm, projection, rotation, attention over [resident cache ; rows], projection,
    norm of the residual's sum, SwiGLU, projection, final norm, cross entropy over the vocabulary
    and the same back, to the rows; their sum over the sequences is the soft prompt's gradient

Random weights and caches stand in for a model's; the optimiser is PyTorch's AdamW.
"""
import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2608_28099_gb300 as sp  # noqa: E402


class ProbeTeacher:
    """A frozen layer over the cache of some sequences, and the soft prompt's loss and gradient."""

    def __init__(self, lens, rows, d_model, n_q_heads, n_kv_heads, head_dim, d_ff, vocab, page=16, theta=1.0e4,
                 eps=1.0e-6, seed=0):
        import torch
        self.torch, self.B, self.k, self.d, self.eps = torch, len(lens), rows, d_model, eps
        self.Hq, self.Hkv, self.dh, self.V = n_q_heads, n_kv_heads, head_dim, vocab
        self.width = (n_q_heads + 2 * n_kv_heads) * head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape, std=1.0: torch.randn(shape, generator=g, device="cuda") * std  # noqa: E731
        weight = lambda out, of: normal(out, of, std=of ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.w_qkv, self.w_o = weight(self.width, d_model), weight(d_model, n_q_heads * head_dim)
        self.w_gu, self.w_down = weight(2 * d_ff, d_model), weight(d_model, d_ff)
        self.back = {n: getattr(self, n).t().contiguous() for n in ("w_qkv", "w_o", "w_gu", "w_down")}
        self.g_in, self.g_post, self.g_final = (1 + normal(d_model, std=0.1) for _ in range(3))
        self.head = weight(vocab, d_model)

        pages = [-(-n // page) for n in lens]
        order = torch.randperm(sum(pages), generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((self.B, max(max(pages), 1)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (max(at, 1), n_kv_heads, page, head_dim)
        self.k_pool, self.v_pool = (normal(*shape).to(torch.bfloat16) for _ in range(2))
        kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, self.k_pool.data_ptr(), self.v_pool.data_ptr(),
                            self.table.data_ptr(), page, shape[0], self.table.shape[1], self.B)
        self.cache = sp.sp_token_cache(kv, sp.SP_BF16, n_kv_heads, head_dim, max(max(lens), 1), None, None)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.pos = (self.lens[:, None] + torch.arange(rows, device="cuda")[None]).to(torch.int32).flatten().contiguous()

        turns, amplitude = sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, head_dim, theta)
        self.turns = torch.from_numpy(turns.view(np.int64)).cuda()
        self.rot = sp.sp_rotary(head_dim, head_dim, 0, amplitude, self.turns.data_ptr())
        n = self.B * rows
        self.tree = sp.sp_tree_dims(n_q_heads, rows, sp.SP_BF16, 0, 0, 0.0, self.width, self.width, self.width)
        self.norm = sp.sp_norm_dims(n, d_model, sp.SP_F32, sp.SP_F32, eps, 0, 0, 0, 0)
        self.loss_dims = sp.sp_vocab_dims(self.B, vocab, d_model, sp.SP_BF16, 0, 0, 0)
        sizes = [sp.sp_attend_tree_workspace_bytes(self.tree, self.cache, self.B),
                 sp.sp_attend_tree_backward_workspace_bytes(self.tree, self.cache, self.B),
                 sp.sp_vocab_loss_workspace_bytes(self.loss_dims), sp.sp_vocab_loss_backward_workspace_bytes(self.loss_dims)]
        for w in (self.w_qkv, self.w_o, self.w_gu, self.w_down):
            sizes += [sp.sp_project_workspace_bytes(n, *w.shape), sp.sp_project_workspace_bytes(n, *w.shape[::-1])]
        if 0 in sizes[:4]:
            raise sp.SpError(0, sp.sp_last_error())
        self.ws_bytes = max(sizes)  # (one call after another on one stream: they share it)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _stream(self):
        return self.torch.cuda.current_stream()

    def _new(self, *shape, dtype=None):
        return self.torch.empty(shape, dtype=dtype or self.torch.float32, device="cuda")

    def _project(self, x, w):
        """x [n][in] (fp32) W^T for W [out][in] (bf16)."""
        y = self._new(x.shape[0], w.shape[0])
        sp.sp_project(self._stream(), x.shape[0], w.shape[0], w.shape[1], x, w, y, 0, self.ws, self.ws_bytes)
        return y

    def _normed(self, x, residual, gain):
        """(the rows' sum, its norm)"""
        total, y = self._new(*x.shape), self._new(*x.shape)
        sp.sp_norm(self._stream(), self.norm, x, residual, gain, total, y)
        return total, y

    def _norm_back(self, grad, total, gain, beside):
        out = self._new(*total.shape)
        sp.sp_norm_backward(self._stream(), self.norm, grad, total, gain, beside, out)
        return out

    def _rotate(self, rows, backward):
        sp.sp_rotate(self._stream(), self.rot, len(rows), self.pos, backward, sp.SP_BF16, self.Hq + self.Hkv, rows,
                     self.width, self.dh, rows, self.width, self.dh)

    def _parts(self, rows):
        q, k = self.Hq * self.dh, self.Hkv * self.dh
        return rows[:, :q], rows[:, q:q + k], rows[:, q + k:]

    def loss_and_gradient(self, prompt, targets):
        """prompt [rows][d] (fp32), targets [B] (int32, negative: none): losses [B] and the mean's gradient."""
        torch, B, n = self.torch, self.B, self.B * self.k
        bf16 = torch.bfloat16
        # ---- forward
        x = prompt.detach().repeat(B, 1)
        _, n1 = self._normed(x, None, self.g_in)
        rows = self._project(n1, self.w_qkv).to(bf16)
        self._rotate(rows, 0)
        o, lse = self._new(n, self.Hq * self.dh, dtype=bf16), self._new(n, self.Hq)
        sp.sp_attend_tree_lse(self._stream(), self.tree, self.cache, B, None, self.lens, None, None, *self._parts(rows), o,
                              lse, self.ws, self.ws_bytes, self.status)
        h1, n2 = self._normed(self._project(o.float(), self.w_o), x, self.g_post)
        gate, up = self._project(n2, self.w_gu).chunk(2, dim=1)
        sig = torch.sigmoid(gate)
        h2, n3 = self._normed(self._project(gate * sig * up, self.w_down), h1, self.g_final)
        last = n3[self.k - 1::self.k].to(bf16).contiguous()  # the rows behind which the label stands
        loss, log_sum = self._new(B), self._new(B)
        sp.sp_vocab_loss(self._stream(), self.loss_dims, last, self.head, targets, loss, log_sum, self.ws, self.ws_bytes,
                         self.status)
        # ---- backward
        with_target = ((targets >= 0).sum().clamp_min(1)).float()
        d_last = self._new(B, self.d, dtype=bf16)
        sp.sp_vocab_loss_backward(self._stream(), self.loss_dims, last, self.head, targets, log_sum,
                                  (torch.ones(B, device="cuda") / with_target), d_last, None, self.ws, self.ws_bytes, self.status)
        d_n3 = torch.zeros(n, self.d, device="cuda")
        d_n3[self.k - 1::self.k] = d_last.float()
        d_h2 = self._norm_back(d_n3, h2, self.g_final, None)
        d_act = self._project(d_h2, self.back["w_down"])
        d_gate = d_act * up * sig * (1 + gate * (1 - sig))
        d_n2 = self._project(torch.cat([d_gate, d_act * gate * sig], 1), self.back["w_gu"])
        d_h1 = self._norm_back(d_n2, h1, self.g_post, d_h2)
        d_o = self._project(d_h1, self.back["w_o"]).to(bf16)
        d_rows = torch.empty_like(rows)
        sp.sp_attend_tree_backward(self._stream(), self.tree, self.cache, B, None, self.lens, None, None, *self._parts(rows),
                                   o, lse, d_o, *self._parts(d_rows), self.ws, self.ws_bytes, self.status)
        self._rotate(d_rows, 1)
        d_x = self._norm_back(self._project(d_rows.float(), self.back["w_qkv"]), x, self.g_in, d_h1)
        return loss, d_x.view(B, self.k, self.d).sum(0)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--lr", type=float, default=3e-2)
    a = ap.parse_args(argv)
    import torch
    rng = np.random.default_rng(0)
    lens = rng.integers(50, 1500, a.batch).tolist()
    t = ProbeTeacher(lens, a.rows, 512, 8, 2, 128, 1024, a.vocab)
    targets = torch.from_numpy(rng.integers(0, a.vocab, a.batch).astype(np.int32)).cuda()
    prompt = torch.nn.Parameter(0.5 * torch.randn(a.rows, t.d, device="cuda"))
    opt = torch.optim.AdamW([prompt], lr=a.lr)
    for step in range(a.steps):
        loss, prompt.grad = t.loss_and_gradient(prompt, targets)
        opt.step()
        if step % 5 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.mean().item():.4f}")
    assert int(t.status) == 0
    return loss


if __name__ == "__main__":
    main()
