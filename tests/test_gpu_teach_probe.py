"""The teaching loop of examples/teach_probe.py: loss and the soft prompt's gradient through
norms, rotation, attention over a cache, SwiGLU and the vocabulary loss, against float64 autograd of
the same layer."""
import importlib.util
import os

import pytest

from conftest import ROOT
from gpu_util import ensure_built, torch_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def load_example():
    spec = importlib.util.spec_from_file_location("teach_probe", os.path.join(ROOT, "examples", "teach_probe.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(torch, t, prompt, targets):
    """Losses and the soft prompt's gradient in float64, from the layer's definition."""
    p = prompt.double().cpu().requires_grad_()
    w = {n: getattr(t, n).double().cpu() for n in ("w_qkv", "w_o", "w_gu", "w_down", "head", "g_in", "g_post", "g_final")}
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + t.eps) * g  # noqa: E731
    turns = t.turns.cpu().double() / 2.0 ** 64  # (frequencies below half a turn: never negative)
    losses = []
    page = t.cache.kv.page_size
    for b in range(t.B):
        L = int(t.lens[b])
        pages = t.table[b, :-(-L // page)].long()
        K, V = (torch.cat([x[i].transpose(0, 1) for i in pages] or [x[0].transpose(0, 1)[:0]])[:L].double().cpu()
                for x in (t.k_pool, t.v_pool))
        rows = (norm(p, w["g_in"]) @ w["w_qkv"].T).view(t.k, -1, t.dh)
        q, k, v = rows[:, :t.Hq], rows[:, t.Hq:t.Hq + t.Hkv], rows[:, t.Hq + t.Hkv:]
        angle = 2 * torch.pi * (L + torch.arange(t.k).double())[:, None] * turns[None]
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        turn = lambda x: torch.cat([x[..., :t.dh // 2] * c - x[..., t.dh // 2:] * s,  # noqa: E731
                                    x[..., t.dh // 2:] * c + x[..., :t.dh // 2] * s], -1)
        q, k = turn(q), torch.cat([K, turn(k)])
        v = torch.cat([V, v])
        sees = torch.cat([torch.ones(t.k, L, dtype=torch.bool), torch.tril(torch.ones(t.k, t.k, dtype=torch.bool))], 1)
        o = []
        for h in range(t.Hq):
            x = (q[:, h] @ k[:, h * t.Hkv // t.Hq].T) * t.dh ** -0.5
            o.append(torch.softmax(x.masked_fill(~sees, -torch.inf), -1) @ v[:, h * t.Hkv // t.Hq])
        h1 = p + torch.cat(o, -1) @ w["w_o"].T
        gate, up = (norm(h1, w["g_post"]) @ w["w_gu"].T).chunk(2, -1)
        h2 = h1 + (torch.nn.functional.silu(gate) * up) @ w["w_down"].T
        logits = w["head"] @ norm(h2[-1], w["g_final"])
        losses.append(torch.logsumexp(logits, 0) - logits[int(targets[b])] if targets[b] >= 0 else (p * 0).sum())
    loss = torch.stack(losses)
    (loss.sum() / (targets >= 0).sum()).backward()
    return loss.detach(), p.grad


@pytest.mark.parametrize("lens,rows,heads", [([70, 0, 300, 1], 4, (4, 2)), ([500, 33], 7, (3, 1)), ([129], 1, (2, 2))])
def test_loss_and_gradient(torch, lens, rows, heads):
    t = load_example().ProbeTeacher(lens, rows, 256, *heads, 128, 256, 300, seed=len(lens))
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randn((rows, t.d), generator=g, device="cuda") * 0.5
    targets = torch.arange(len(lens), dtype=torch.int32, device="cuda") * 7
    if len(lens) > 2:
        targets[2] = -1
    want, grad = reference(torch, t, prompt, targets.cpu())
    loss, got = t.loss_and_gradient(prompt, targets)
    assert int(t.status) == 0
    # bf16 between the calls: q/k/v, weights, attention output, last row and four of the gradients on the way
    # back, 2^-8 of their size each, which the layer passes on at most twofold; losses move by the logits' change
    scale = 8 * 2 * 2.0 ** -8
    assert bool(((loss.cpu().double() - want).abs() <= scale * (1 + want.abs())).all())
    assert float((got.cpu().double() - grad).norm()) <= scale * float(grad.norm())
    again = t.loss_and_gradient(prompt, targets)
    assert torch.equal(again[0], loss) and torch.equal(again[1], got)
    st = torch.cuda.Stream()  # there a call's set-up runs beside the call before it
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        rows = [t.loss_and_gradient(prompt, targets) for _ in range(3)]
    st.synchronize()
    assert all(torch.equal(a, loss) and torch.equal(b, got) for a, b in rows)


def test_the_example_runs(torch):
    loss = load_example().main(["--batch", "4", "--rows", "3", "--steps", "3", "--vocab", "300"])
    assert bool(loss.isfinite().all())
