"""Performance cases of the operators that teach a probe: root-mean-square norm with
the residual's addition (rows or 8-bit rows out) and its backward pass, the backward
pass of the attention over a resident token cache, and the cross entropy over a large
vocabulary, with its gradients, whose logits are never kept.

A case is one call.  Layer shapes are those of the workloads module's draft heads (the
0.6B- to 27B-class ones and the tiny fp32 one); vocabularies are generic.  Cached keys
and values are N(0, 1) with a magnitude of their own for every (token, head), queries
N(0, 0.02 sqrt(d)) like rotated projections, weights N(0, 0.02); hidden states lean to
their token's row of the head, as those of a model that has learnt something do, so that
probabilities of the targets run from nearly none to nearly one.
`own` chooses between the framework's calls and the operators' plain forms in 32-bit
elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

# query heads, kv heads, head_dim, d_model
LAYERS = {
    "tiny": (4, 2, 32, 128),
    "0.6b": (16, 8, 128, 1024),
    "4b": (32, 8, 128, 2560),
    "8b": (32, 8, 128, 4096),
    "27b": (40, 8, 128, 5120),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
EPS = 1.0e-6


def _norm_case(name, n, d, dtype, out, residual=True):
    """n rows of d; out: type of the normed rows (e4m3: codes with a scale a row);
    residual: added first, and the sum is written too."""
    return {"name": name, "op": "norm", "n": n, "d": d, "dtype": dtype, "out": out, "residual": residual}


def _norm_backward_case(name, n, d, dtype, beside=True, gain=True):
    """beside: a gradient that reaches the sum past the norm is added; gain: the
    gain's gradient is wanted."""
    return {"name": name, "op": "norm_backward", "n": n, "d": d, "dtype": dtype, "beside": beside, "gain": gain}


def _attend_case(name, layer, B, lens, nodes, dtype, page, tree=False, ragged=False):
    """nodes: query rows of a sequence (a probe's soft-prompt rows, each seeing those
    before it; tree: drafted nodes with random parents); ragged: some have fewer;
    lens = (fewest, most) cached tokens; page 0 = contiguous."""
    return {"name": name, "op": "attend_backward", "layer": layer, "B": B, "lo": lens[0], "hi": lens[1],
            "nodes": nodes, "dtype": dtype, "page": page, "tree": tree, "ragged": ragged}


def _loss_case(name, n, d, V, dtype, skip=0.0):
    """n tokens of d against V rows; skip: share of the tokens that have no target."""
    return {"name": name, "op": "loss", "n": n, "d": d, "V": V, "dtype": dtype, "skip": skip}


def _loss_backward_case(name, n, d, V, dtype, head, skip=0.0):
    """head: the head's gradient is wanted beside the hidden states'."""
    return {"name": name, "op": "loss_backward", "n": n, "d": d, "V": V, "dtype": dtype, "head": head, "skip": skip}


def listed():
    return [
        # the post-attention norm of one decoding step: launch latency
        _norm_case("norm_step", 16, 4096, "bf16", "bf16"),
        # a prompt's rows into 8 bits, as an 8-bit projection takes them
        _norm_case("norm_prompt_8bit", 16384, 5120, "bf16", "e4m3"),
        # a training step's rows, odd in number, with the gain's gradient
        _norm_backward_case("norm_backward", 8191, 4096, "bf16"),
        # the same in fp32, the layer frozen
        _norm_backward_case("norm_backward_frozen", 1500, 2560, "f32", gain=False),
        # a soft prompt trained on one document
        _attend_case("attend_backward_one", "8b", 1, (2048, 2048), 8, "bf16", 16),
        # the 8B-class batch of documents, 16 soft-prompt rows
        _attend_case("attend_backward_8b", "8b", 64, (1024, 8192), 16, "bf16", 16),
        # the 27B-class long-context batch
        _attend_case("attend_backward_27b", "27b", 8, (32768, 32768), 16, "bf16", 16),
        # one answer's tokens scored: the weights are read once
        _loss_case("loss_answer", 48, 2560, 32000, "bf16"),
        # a training step's loss, a third of the tokens without a target
        _loss_case("loss_train", 4096, 4096, 65536, "bf16", skip=0.33),
        # gradients of the hidden states under a frozen head
        _loss_backward_case("loss_backward_frozen", 4096, 4096, 65536, "bf16", False, skip=0.33),
        # with the head's gradient, odd token count and vocabulary
        _loss_backward_case("loss_backward_head", 2051, 2560, 50021, "bf16", True),
        # the tiny fp32 layer (everything in 32 bits)
        _loss_backward_case("loss_backward_fp32", 250, 128, 1000, "f32", True),
    ]


def _cost(case):
    """A rough time of a call, to bound the drawn ones (fp32 work runs on CUDA cores)."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (2e13 if case["dtype"] == "f32" else 1e15)


def _log(rng, lo, hi):
    return int(round(2 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    """One more call of the same ranges."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choice(["norm", "norm_backward", "attend_backward", "attend_backward", "loss", "loss_backward"])
        d = rng.choice([1024, 2560, 4096, 5120, _log(rng, 16, 1024) * 8])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        if op == "norm":
            c = _norm_case("", _log(rng, 1, 20000), d, dtype, rng.choice([dtype, dtype, "e4m3"]), rng.random() < 0.7)
        elif op == "norm_backward":
            c = _norm_backward_case("", _log(rng, 1, 10000), d, dtype, rng.random() < 0.6, rng.random() < 0.6)
        elif op == "attend_backward":
            hi = _log(rng, 16, 32768)
            layer = rng.choice(["tiny", "0.6b"]) if dtype == "f32" else rng.choice(["0.6b", "4b", "8b", "8b", "27b"])
            c = _attend_case("", layer, _log(rng, 1, 128), (int(hi * rng.choice([0.0, 0.3, 1.0])), hi),
                             _log(rng, 1, 32), dtype, rng.choice([0, 16, 16, 32, 64]), rng.random() < 0.3,
                             rng.random() < 0.4)
        else:
            n, V = _log(rng, 1, 8192), _log(rng, 300, 130000)
            if dtype == "f32":
                d, n, V = _log(rng, 2, 64) * 8, _log(rng, 1, 500), _log(rng, 2, 4000)
            skip = rng.choice([0.0, 0.0, 0.2, 0.6])
            c = _loss_case("", n, d, V, dtype, skip) if op == "loss" else _loss_backward_case(
                "", n, d, V, dtype, rng.random() < 0.5, skip)
        if _cost(c) <= most[op]:
            del c["name"]
            return c


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _generators(seed):
    g, h = torch.Generator(device="cuda"), torch.Generator()
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    h.manual_seed((int(seed) ^ 0x5DEECE66D) & 0x7FFFFFFFFFFF)
    return g, h


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)


def _int(h, lo, hi, shape):
    """Uniform integers lo..hi."""
    return torch.randint(lo, hi + 1, shape, generator=h, dtype=torch.int32)


def _draw_cache(case, g, h, lens):
    """K, V [page][Hkv][P][dh] with a random page table, or [slots][Hkv][dh]."""
    _, hkv, dh, _ = LAYERS[case["layer"]]
    P, most = case["page"], max(case["hi"], 1)
    c = {}
    if P:
        pages = (lens + P - 1) // P
        table = torch.full((len(lens), (most + P - 1) // P), -1, dtype=torch.int32)
        used = torch.arange(table.shape[1])[None] < pages[:, None]
        total = table.numel()
        table[used] = torch.randperm(total, generator=h)[:int(pages.sum())].to(torch.int32)
        c["table"] = table.cuda()
        shape, at = (total, hkv, P, dh), (total, hkv, P)
    else:
        c["start"] = (torch.cumsum(lens, 0) - lens).to(torch.int64).cuda()
        shape, at = (len(lens) * most, hkv, dh), (len(lens) * most, hkv)
    for n in ("k", "v"):
        x = _normal(g, shape)
        x *= torch.exp(0.3 * _normal(g, at))[..., None]
        c[n] = x.to(DTYPES[case["dtype"]])
        del x
    return c


def _draw_masks(h, B, N, tree, ragged):
    """Masks [B][N] (bit j: row i sees row j) and row counts [B]: each sees itself and
    those before it, or, in a tree, those above it; a row past the count sees nothing."""
    n = _int(h, max(1, N // 2), N, (B,)) if ragged else torch.full((B,), N, dtype=torch.int32)
    mask = torch.zeros((B, N), dtype=torch.int64)
    up = torch.randint(0, 1 << 30, (B, N), generator=h) % (torch.arange(N)[None] + 1) - 1
    if not tree:
        up = torch.arange(N)[None].expand(B, N) - 1
    for i in range(N):
        above = mask.gather(1, up[:, i:i + 1].clamp_min(0))[:, 0]
        mask[:, i] = torch.where(up[:, i] >= 0, above, torch.zeros_like(above)) | (1 << i)
    mask[torch.arange(N)[None] >= n[:, None]] = 0
    return mask, n


def _draw(case, seed):
    g, h = _generators(seed)
    dt = DTYPES[case["dtype"]]
    op = case["op"]
    s = {}
    if op in ("norm", "norm_backward"):
        n, d = case["n"], case["d"]
        size = torch.exp(0.5 * _normal(g, (n, 1)))
        s["x"] = (_normal(g, (n, d)) * size).to(dt)
        s["gain"] = 1.0 + _normal(g, (d,), 0.1)
        if op == "norm":
            s["r"] = (_normal(g, (n, d), 0.5) * size).to(dt) if case["residual"] else None
        else:
            s["dy"] = _normal(g, (n, d), 0.01).to(dt)
            s["ds"] = _normal(g, (n, d), 0.01).to(dt) if case["beside"] else None
        return s
    if op == "attend_backward":
        hq, hkv, dh, d = LAYERS[case["layer"]]
        B, N, spread = case["B"], case["nodes"], 0.02 * math.sqrt(d)
        lens = _int(h, case["lo"], case["hi"], (B,)).to(torch.int64)
        s["lens"] = lens.to(torch.int32).cuda()
        s["cache"] = _draw_cache(case, g, h, lens)
        s["longest"] = max(case["hi"], 1)
        s["q"] = _normal(g, (B, N, hq, dh), spread).to(dt)
        s["k_new"] = _normal(g, (B, N, hkv, dh)).to(dt)
        s["v_new"] = _normal(g, (B, N, hkv, dh)).to(dt)
        s["do"] = _normal(g, (B, N, hq, dh), 0.01).to(dt)
        mask, n = _draw_masks(h, B, N, case["tree"], case["ragged"])
        s["mask"], s["n"] = mask.cuda(), n.cuda()
        return s
    n, d, V = case["n"], case["d"], case["V"]
    s["w"] = _normal(g, (V, d), 0.02).to(dt)
    t = _int(h, 0, V - 1, (n,))
    t[torch.rand(n, generator=h) < case["skip"]] = -1
    s["t"] = t.cuda()
    lean = 8.0 * torch.rand(n, generator=g, device="cuda") * 4096.0 / d
    x = _normal(g, (n, d))
    x += lean[:, None] * s["w"][s["t"].clamp_min(0).long()].to(torch.float32)
    s["h"] = x.to(dt)
    if op == "loss_backward":
        s["dloss"] = (torch.rand(n, generator=g, device="cuda") + 0.5) / n
    return s


_STREAM = None


def _stream():
    """The program's own stream (calls on it overlap their set-up)."""
    global _STREAM
    if _STREAM is None:
        _STREAM = torch.cuda.Stream()
    return _STREAM


def _plan(case, s):
    """What a program keeps between calls: descriptors, outputs, workspace."""
    import paper_2608_28099_gb300 as sp
    dt = {"f32": sp.SP_F32, "bf16": sp.SP_BF16, "e4m3": sp.SP_E4M3}
    p, op, T = {"sp": sp}, case["op"], DTYPES[case["dtype"]]
    new = lambda shape, t=T: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    size = 0
    if op in ("norm", "norm_backward"):
        n, d = case["n"], case["d"]
        p["dims"] = sp.sp_norm_dims(n, d, dt[case["dtype"]], dt[case.get("out", case["dtype"])], EPS, 0, 0, 0, 0)
        if op == "norm":
            p["y"] = new((n, d), DTYPES[case["out"]])
            p["scale"] = new((n,), torch.float32) if case["out"] == "e4m3" else None
            p["sum"] = new((n, d)) if case["residual"] else None
        else:
            p["dx"] = new((n, d))
            p["dgain"] = new((d,), torch.float32) if case["gain"] else None
            size = sp.sp_norm_backward_workspace_bytes(p["dims"])
    elif op == "attend_backward":
        hq, hkv, dh, _ = LAYERS[case["layer"]]
        c, B, P, N = s["cache"], case["B"], case["page"], case["nodes"]
        if P:
            kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, c["k"].data_ptr(), c["v"].data_ptr(),
                                c["table"].data_ptr(), P, c["k"].shape[0], c["table"].shape[1], B)
        else:
            step = hkv * dh * c["k"].element_size()
            p["at"] = [c[n].data_ptr() + c["start"] * step for n in ("k", "v")]
            kv = sp.sp_kv_cache(sp.SP_KV_CONTIGUOUS, p["at"][0].data_ptr(), p["at"][1].data_ptr(), None, None, None,
                                0, 0, 0, B)
        p["cache"] = sp.sp_token_cache(kv, dt[case["dtype"]], hkv, dh, s["longest"], None, None)
        p["dims"] = sp.sp_tree_dims(hq, N, dt[case["dtype"]], 0, 0, 0.0, 0, 0, 0)
        p["dq"], p["dk"], p["dv"] = new((B, N, hq, dh)), new((B, N, hkv, dh)), new((B, N, hkv, dh))
        size = sp.sp_attend_tree_backward_workspace_bytes(p["dims"], p["cache"], B)
    else:
        n, d, V = case["n"], case["d"], case["V"]
        p["dims"] = sp.sp_vocab_dims(n, V, d, dt[case["dtype"]], 0, 0, 0)
        if op == "loss":
            p["loss"], p["lse"] = new((n,), torch.float32), new((n,), torch.float32)
            size = sp.sp_vocab_loss_workspace_bytes(p["dims"])
        else:
            p["dh"] = new((n, d))
            p["dw"] = new((V, d)) if case["head"] else None
            size = sp.sp_vocab_loss_backward_workspace_bytes(p["dims"])
    p["bytes"] = size
    p["ws"] = new((max(size, 1),), torch.uint8)
    return p


def prepare(case, seed):
    s = _draw(case, seed)
    s["case"] = case
    # what the forward pass has left: the attention's output and log sums, the loss's log sums
    if case["op"] == "attend_backward":
        s["o"], s["lse"] = _plain_attend(s)[:2]
    elif case["op"] == "loss_backward":
        s["lse"] = _plain_loss(s)[1]
    if own:
        s["plan"] = _plan(case, s)
    torch.cuda.synchronize()
    return s


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def run(s):
    return _call(s) if own else {"norm": _plain_norm, "norm_backward": _plain_norm_backward,
                                 "attend_backward": _plain_attend_backward, "loss": _plain_loss,
                                 "loss_backward": _plain_loss_backward}[s["case"]["op"]](s)


def _call(s):
    case, p, st = s["case"], s["plan"], _stream()
    sp, op, dims = p["sp"], case["op"], p["dims"]
    if op == "norm":
        sp.sp_norm(st, dims, s["x"], s["r"], s["gain"], p["sum"], p["y"], p["scale"])
        return [t for t in (p["y"], p["scale"], p["sum"]) if t is not None]
    if op == "norm_backward":
        sp.sp_norm_backward(st, dims, s["dy"], s["x"], s["gain"], s["ds"], p["dx"], p["dgain"], p["ws"], p["bytes"])
        return [t for t in (p["dx"], p["dgain"]) if t is not None]
    if op == "attend_backward":
        sp.sp_attend_tree_backward(st, dims, p["cache"], case["B"], None, s["lens"], s["mask"], s["n"], s["q"],
                                   s["k_new"], s["v_new"], s["o"], s["lse"], s["do"], p["dq"], p["dk"], p["dv"],
                                   p["ws"], p["bytes"])
        return [p["dq"], p["dk"], p["dv"]]
    if op == "loss":
        sp.sp_vocab_loss(st, dims, s["h"], s["w"], s["t"], p["loss"], p["lse"], p["ws"], p["bytes"])
        return [p["loss"], p["lse"]]
    sp.sp_vocab_loss_backward(st, dims, s["h"], s["w"], s["t"], s["lse"], s["dloss"], p["dh"], p["dw"], p["ws"],
                              p["bytes"])
    return [t for t in (p["dh"], p["dw"]) if t is not None]


def _plain_norm(s):
    dt, out = DTYPES[s["case"]["dtype"]], s["case"]["out"]
    x = s["x"].to(torch.float32)
    x = x + s["r"].to(torch.float32) if s["r"] is not None else x
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain"]
    if out == "e4m3":
        amax = y.abs().amax(-1).clamp_min(2.0 ** -60)
        got = [(y * (torch.full_like(amax, 448.0) / amax)[:, None]).to(torch.float8_e4m3fn), amax * (1.0 / 448.0)]
    else:
        got = [y.to(DTYPES[out])]
    return got + ([x.to(dt)] if s["r"] is not None else [])


def _plain_norm_backward(s):
    case = s["case"]
    x, dy = s["x"].to(torch.float32), s["dy"].to(torch.float32)
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    x = x * rstd
    gy = dy * s["gain"]
    dx = rstd * (gy - x * (gy * x).mean(-1, keepdim=True))
    dx = (dx + s["ds"].to(torch.float32) if case["beside"] else dx).to(s["x"].dtype)
    return [dx, (dy * x).sum(0)] if case["gain"] else [dx]


def _plain_gather(s, n):
    """Keys or values [B][longest][Hkv][dh] in fp32, zero past each sequence's end."""
    c, case = s["cache"], s["case"]
    T = s["longest"]
    if case["page"]:
        x = c[n][c["table"].to(torch.int64).clamp_min(0)].transpose(2, 3).flatten(1, 2)[:, :T]
    else:
        at = (c["start"][:, None] + torch.arange(T, device="cuda")[None]).clamp_max(c[n].shape[0] - 1)
        x = c[n][at]
    inside = torch.arange(T, device="cuda")[None] < s["lens"][:, None]
    return torch.where(inside[:, :, None, None], x.to(torch.float32), torch.zeros((), device="cuda"))


def _plain_attend(s):
    """The forward pass: output [B][N][Hq][dh] (rounded), log sums [B][N][Hq], and what
    the backward pass needs again: weights, keys, values, queries [B][Hkv][...]."""
    case = s["case"]
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    B, N, T, G = case["B"], case["nodes"], s["longest"], hq // hkv
    alive = torch.arange(N, device="cuda")[None] < s["n"][:, None]
    rows = lambda x: x.to(torch.float32).view(B, N, hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * G, dh)  # noqa: E731
    q = rows(s["q"])
    fresh = [torch.where(alive[:, :, None, None], s[n].to(torch.float32), torch.zeros((), device="cuda"))
             for n in ("k_new", "v_new")]
    k, v = (torch.cat([_plain_gather(s, n), f], 1).permute(0, 2, 1, 3) for n, f in zip(("k", "v"), fresh))
    sees = ((s["mask"][:, :, None] >> torch.arange(N, device="cuda")) & 1).to(torch.bool) & alive[:, :, None] & alive[:, None]
    inside = (torch.arange(T, device="cuda")[None] < s["lens"][:, None])[:, None] & alive[:, :, None]
    sees = torch.cat([inside, sees], 2).repeat_interleave(G, 1)[:, None]
    p = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(dh))
    p = p.masked_fill_(~sees, -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp_(p.sub_(top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p /= torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v).view(B, hkv, N, G, dh).permute(0, 2, 1, 3, 4).reshape(B, N, hq, dh)
    lse = lse.view(B, hkv, N, G).permute(0, 2, 1, 3).reshape(B, N, hq).contiguous()
    return o.to(s["q"].dtype), lse, p, k, v, q, rows


def _plain_attend_backward(s):
    case = s["case"]
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    B, N, T, G, dt = case["B"], case["nodes"], s["longest"], hq // hkv, s["q"].dtype
    _, _, p, k, v, q, rows = _plain_attend(s)
    do = rows(s["do"])
    dv = torch.matmul(p[..., T:].transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2))
    ds -= (ds * p).sum(-1, keepdim=True)
    ds *= p
    ds *= 1.0 / math.sqrt(dh)
    dq = torch.matmul(ds, k).view(B, hkv, N, G, dh).permute(0, 2, 1, 3, 4).reshape(B, N, hq, dh)
    dk = torch.matmul(ds[..., T:].transpose(-1, -2), q)
    return [dq.to(dt)] + [x.transpose(1, 2).to(dt).contiguous() for x in (dk, dv)]


def _pieces(s):
    """The vocabulary a piece at a time: (first row, rows in fp32)."""
    step = 8192
    for v in range(0, s["w"].shape[0], step):
        yield v, s["w"][v:v + step].to(torch.float32)


def _plain_loss(s):
    h, t = s["h"].to(torch.float32), s["t"].to(torch.int64)
    top = torch.full((h.shape[0],), -math.inf, device="cuda")
    total, at = torch.zeros_like(top), torch.zeros_like(top)
    for v, w in _pieces(s):
        x = torch.matmul(h, w.T)
        new = torch.maximum(top, x.amax(-1))
        total = total * torch.exp(top - new) + torch.exp(x - new[:, None]).sum(-1)
        top = new
        here = (t >= v) & (t < v + w.shape[0])
        at = torch.where(here, x.gather(1, (t - v).clamp(0, w.shape[0] - 1)[:, None])[:, 0], at)
    lse = top + torch.log(total)
    zero = torch.zeros((), device="cuda")
    return [torch.where(t >= 0, lse - at, zero), torch.where(t >= 0, lse, zero)]


def _plain_loss_backward(s):
    h, t, dt = s["h"].to(torch.float32), s["t"].to(torch.int64), s["h"].dtype
    dloss = torch.where(t >= 0, s["dloss"], torch.zeros((), device="cuda"))
    dh = torch.zeros_like(h)
    dw = torch.empty_like(s["w"]) if s["case"]["head"] else None
    for v, w in _pieces(s):
        g = torch.exp(torch.matmul(h, w.T) - s["lse"][:, None])
        here = ((t >= v) & (t < v + w.shape[0])).nonzero()[:, 0]
        g[here, t[here] - v] -= 1.0
        g *= dloss[:, None]
        g = torch.where((t >= 0)[:, None], g, torch.zeros((), device="cuda"))
        dh += torch.matmul(g, w)
        if dw is not None:
            dw[v:v + w.shape[0]] = torch.matmul(g.T, h).to(dt)
    return [dh.to(dt)] + ([dw] if dw is not None else [])


# --------------------------------------------------------------------------- #
# what a pass cannot do without
# --------------------------------------------------------------------------- #
def work(case):
    e, op = BYTES[case["dtype"]], case["op"]
    if op == "norm":
        rows = case["n"] * case["d"]
        moved = rows * ((3 if case["residual"] else 1) * e + BYTES[case["out"]])
        return {"bytes": moved + 4.0 * case["d"], "flops": 5.0 * rows}
    if op == "norm_backward":
        rows = case["n"] * case["d"]
        return {"bytes": rows * (3.0 + case["beside"]) * e + (8.0 if case["gain"] else 4.0) * case["d"], "flops": 9.0 * rows}
    if op == "attend_backward":
        hq, hkv, dh, _ = LAYERS[case["layer"]]
        cached, rows = case["B"] * (case["lo"] + case["hi"]) / 2.0, case["B"] * case["nodes"]
        live = rows * (0.75 if case["ragged"] else 1.0)
        # scores, the weights' gradients and the queries' gradients over the cache; the rows' own
        # keys and values take two products more
        return {"bytes": cached * 2.0 * hkv * dh * e + rows * (dh * e * 4.0 * (hq + hkv) + 4.0 * hq + 8),
                "flops": 6.0 * dh * hq * live * cached / case["B"] + 5.0 * dh * hq * live * case["nodes"]}
    kept = case["n"] * (1.0 - case["skip"])
    product = 2.0 * kept * case["d"] * case["V"]
    once = (kept * case["d"] + case["V"] * case["d"]) * e + 12.0 * case["n"]
    if op == "loss":
        return {"bytes": once, "flops": product + 3.0 * kept * case["V"]}
    out = (case["n"] * case["d"] + (case["V"] * case["d"] if case["head"] else 0)) * e
    return {"bytes": once + out, "flops": product * (3 if case["head"] else 2) + 3.0 * kept * case["V"]}


# --------------------------------------------------------------------------- #
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------- #
def _e4m3_64(x):
    """Nearest value of 1 sign, 4 exponent (bias 7) and 3 mantissa bits, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _cached64(case, s, b, n):
    """Keys or values [L][Hkv][dh] of sequence b."""
    c, L, P = s["cache"], int(s["lens"][b]), case["page"]
    if not P:
        o = int(c["start"][b])
        return c[n][o:o + L].double()
    pages = c["table"][b, :-(-L // P)].long()
    x = torch.cat([c[n][int(i)].transpose(0, 1) for i in pages] or [c[n][0].transpose(0, 1)[:0]])
    return x[:L].double()


def _exact_attend(case, s):
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    B, N, G = case["B"], case["nodes"], hq // hkv
    dq = torch.zeros((B, N, hq, dh), dtype=torch.float64, device="cuda")
    dk, dv = (torch.zeros((B, N, hkv, dh), dtype=torch.float64, device="cuda") for _ in range(2))
    bits = torch.arange(64, device="cuda")
    for b in range(B):
        n, L = int(s["n"][b]), int(s["lens"][b])
        K, V = (torch.cat([_cached64(case, s, b, c), s[c + "_new"][b, :n].double()]) for c in ("k", "v"))
        sees = torch.ones((n, L + n), dtype=torch.bool, device="cuda")
        sees[:, L:] = ((s["mask"][b, :n, None] >> bits) & 1)[:, :n].bool()
        for hh in range(hq):
            k, v = K[:, hh // G], V[:, hh // G]
            q, do = s["q"][b, :n, hh].double(), s["do"][b, :n, hh].double()
            p = torch.softmax((q @ k.T / math.sqrt(dh)).masked_fill(~sees, -math.inf), -1)
            dp = do @ v.T
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(dh)
            dq[b, :n, hh] = ds @ k
            dk[b, :n, hh // G] += ds[:, L:].T @ q
            dv[b, :n, hh // G] += p[:, L:].T @ do
    return [dq, dk, dv]


def exact(case, seed):
    op = case["op"]
    if op in ("loss", "loss_backward") and work(case)["flops"] > 8e12:
        return None  # (64-bit products of that size take too long)
    s = _draw(case, seed)
    if op == "norm":
        x = s["x"].double() + (s["r"].double() if case["residual"] else 0.0)
        y = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * s["gain"].double()
        got = [y]
        if case["out"] == "e4m3":
            scale = y.abs().amax(-1).clamp_min(2.0 ** -60) / 448.0
            got = [_e4m3_64(y / scale[:, None]), scale]
        return got + ([x] if case["residual"] else [])
    if op == "norm_backward":
        x, g, dy, d = s["x"].double(), s["gain"].double(), s["dy"].double(), case["d"]
        ms = torch.mean(x ** 2, -1, keepdim=True) + EPS
        dx = dy * g / torch.sqrt(ms) - x * torch.sum(dy * g * x, -1, keepdim=True) / (d * ms ** 1.5)
        dx = dx + s["ds"].double() if case["beside"] else dx
        return [dx, torch.sum(dy * x / torch.sqrt(ms), 0)] if case["gain"] else [dx]
    if op == "attend_backward":
        return _exact_attend(case, s)
    # a block of tokens at a time: 64-bit logits of all of them would not fit
    w, t, n = s["w"].double(), s["t"].long(), case["n"]
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dh = torch.zeros((n, case["d"]), dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w) if case.get("head") else None
    for a in range(0, n, 512):
        keep = a + (t[a:a + 512] >= 0).nonzero()[:, 0]
        x = s["h"][keep].double()
        logits = x @ w.T
        hot = torch.arange(len(keep), device="cuda"), t[keep]
        lse[keep] = torch.logsumexp(logits, -1)
        loss[keep] = lse[keep] - logits[hot]
        if op == "loss":
            continue
        p = torch.softmax(logits, -1)
        p[hot] -= 1.0
        p *= s["dloss"][keep].double()[:, None]
        dh[keep] = p @ w
        if dw is not None:
            dw += p.T @ x
    return [loss, lse] if op == "loss" else [dh] + ([dw] if dw is not None else [])
