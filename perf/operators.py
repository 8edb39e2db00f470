"""Performance cases of the token-cache operators: rotary positions, appending to
and reading from a (quantised) token cache, and the attention of a tree of
drafted tokens over it.

A case is one call.  Head shapes are those of the workloads module's draft heads
(the 0.6B- to 27B-class ones and the tiny fp32 one); cached keys and values are
N(0, 1) with a magnitude of their own for every (token, head), as projections of
real hidden states have it, queries N(0, 0.02 sqrt(d)) like rotated projections.
`own` chooses between the framework's calls and the operators' plain forms in
32-bit elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

# query heads, kv heads, head_dim, d_model (the queries' spread)
LAYERS = {
    "tiny": (4, 2, 32, 128),
    "0.6b": (16, 8, 128, 1024),
    "4b": (32, 8, 128, 2560),
    "8b": (32, 8, 128, 4096),
    "27b": (40, 8, 128, 5120),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
THETA = 1.0e4


def _rotate_case(name, n, layer, dtype, pairs=False, rot=0, scaling="none", far=8192, backward=False):
    """n tokens of the query and key heads of a fused projection (value heads
    behind them in each row); pairs: interleaved layout; rot: rotated dims (0 =
    all); far: positions 0..far; backward: gradients instead of activations."""
    return {"name": name, "op": "rotate", "n": n, "layer": layer, "dtype": dtype, "pairs": pairs,
            "rot": rot, "scaling": scaling, "far": far, "backward": backward}


def _append_case(name, layer, B, rows, lens, cache, dtype, page, rope, take=0):
    """rows = (fewest, most) new tokens a sequence, lens = (fewest, most) cached
    ones; page 0 = contiguous; take: the appended tokens are a path through a
    drafted tree of that many nodes, 0 = consecutive rows."""
    return {"name": name, "op": "append", "layer": layer, "B": B, "new_lo": rows[0], "new_hi": rows[1],
            "lo": lens[0], "hi": lens[1], "cache": cache, "dtype": dtype, "page": page, "rope": rope,
            "take": take}


def _read_case(name, layer, B, lens, cache, dtype, page):
    return {"name": name, "op": "read", "layer": layer, "B": B, "lo": lens[0], "hi": lens[1], "cache": cache,
            "dtype": dtype, "page": page}


def _tree_case(name, layer, B, lens, nodes, cache, dtype, page, ragged=False):
    """nodes: drafted tokens of a sequence (ragged: some trees are smaller)."""
    return {"name": name, "op": "tree", "layer": layer, "B": B, "lo": lens[0], "hi": lens[1], "nodes": nodes,
            "cache": cache, "dtype": dtype, "page": page, "ragged": ragged}


def listed():
    return [
        # one decoding step of a small batch: launch latency
        _rotate_case("rotate_step", 16, "8b", "bf16"),
        # a prompt's queries and keys, half of the head rotated, a context
        # stretched past the trained one
        _rotate_case("rotate_prompt", 16384, "27b", "bf16", pairs=True, rot=64, scaling="dims", far=131071),
        # the backward pass of a training step in fp32, odd token count
        _rotate_case("rotate_backward", 4099, "8b", "f32", scaling="turns", far=65535, backward=True),
        # the accepted paths of a verified batch written into an 8-bit cache
        _append_case("append_accepted", "8b", 64, (0, 6), (200, 1500), "e4m3", "bf16", 16, False, take=16),
        # a prefill's keys and values: rotated and quantised as they are written
        _append_case("append_prompts", "8b", 12, (500, 4000), (0, 300), "e4m3", "bf16", 16, True),
        # a few short contexts back in fp32, for inspection
        _read_case("read_short", "4b", 3, (100, 700), "e4m3", "f32", 0),
        # long contexts handed to a consumer that wants bf16
        _read_case("read_long", "8b", 6, (3000, 9000), "e4m3", "bf16", 16),
        # one request with a small tree: latency
        _tree_case("tree_one", "8b", 1, (2048, 2048), 8, "bf16", "bf16", 16),
        # the 8B-class serving batch, bf16 cache
        _tree_case("tree_8b_paged", "8b", 64, (1024, 8192), 16, "bf16", "bf16", 16, ragged=True),
        # the 27B-class long-context batch, 8-bit cache, a large tree
        _tree_case("tree_27b_long", "27b", 8, (32768, 32768), 32, "e4m3", "bf16", 16),
        # plain decoding: one token a sequence, 8-bit contiguous caches
        _tree_case("tree_token", "4b", 128, (300, 4000), 1, "e4m3", "bf16", 0),
        # the tiny fp32 layer (everything in 32 bits)
        _tree_case("tree_fp32", "tiny", 5, (0, 500), 11, "f32", "f32", 16, ragged=True),
    ]


def _cost(case):
    """A rough time of a call, to bound the drawn ones (fp32 work runs on CUDA cores)."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (2e13 if case["dtype"] == "f32" else 1e15)


def _log(rng, lo, hi):
    return int(round(2 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    """One more call of the same ranges."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["rotate", "append", "read", "tree", "tree", "tree"])
        layer = rng.choice(["0.6b", "4b", "8b", "8b", "27b"])
        page = rng.choice([0, 16, 16, 32, 64])
        if op == "rotate":
            c = _rotate_case("", _log(rng, 1, 20000), layer, rng.choice(["bf16", "bf16", "f32"]),
                             rng.random() < 0.5, rng.choice([0, 0, 32, 64]),
                             rng.choice(["none", "linear", "base", "turns", "dims"]), _log(rng, 100, 1 << 20),
                             rng.random() < 0.4)
        elif op == "append":
            take = rng.choice([0, 0, 8, 33])
            most_new = min(take, 9) if take else _log(rng, 1, 5000)
            cache = rng.choice(["e4m3", "e4m3", "bf16"])
            c = _append_case("", layer, _log(rng, 1, 100), (rng.randint(0, most_new), most_new),
                             (0, _log(rng, 1, 2000)), cache, rng.choice(["bf16", "bf16", "f32"]), page,
                             not take and rng.random() < 0.7, take)
        elif op == "read":
            hi = _log(rng, 1, 10000)
            c = _read_case("", layer, _log(rng, 1, 64), (rng.randint(0, hi), hi), rng.choice(["e4m3", "e4m3", "bf16"]),
                           rng.choice(["bf16", "f32"]), page)
        else:
            hi = _log(rng, 16, 32768)
            wide = rng.random() < 0.15
            c = _tree_case("", rng.choice(["tiny", "0.6b"]) if wide else layer, _log(rng, 1, 200),
                           (int(hi * rng.choice([0.0, 0.3, 1.0])), hi), _log(rng, 1, 64),
                           "f32" if wide else rng.choice(["bf16", "e4m3"]), "f32" if wide else "bf16", page,
                           rng.random() < 0.5)
        if _cost(c) <= most and (op != "append" or c["B"] * (c["hi"] + c["new_hi"]) <= 150000):
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


def _scaling(case, rot):
    """(kind, factor, trained length, fewest turns, most turns) of a case's rotary."""
    return {"none": ("none", 1.0, 0, 0.0, 0.0), "linear": ("linear", 8.0, 0, 0.0, 0.0),
            "base": ("base", 4.0, 0, 0.0, 0.0), "turns": ("turns", 8.0, 8192, 1.0, 4.0),
            "dims": ("dims", 16.0, 8192, 1.0, 32.0)}[case.get("scaling", "none")]


def _turns(case, rot):
    """The rotation of one position, as 64-bit fixed-point fractions of a turn
    [rot / 2], and the amplitude: the table that a program lays out once."""
    kind, factor, trained, few, many = _scaling(case, rot)
    theta = THETA * factor ** (rot / (rot - 2)) if kind == "base" else THETA
    f = [theta ** (-2.0 * i / rot) / (2.0 * math.pi) for i in range(rot // 2)]
    amplitude = 1.0
    if kind == "linear":
        f = [x / factor for x in f]
    elif kind == "turns":
        w = [min(max((trained * x - few) / (many - few), 0.0), 1.0) for x in f]
        f = [a * x + (1.0 - a) * x / factor for a, x in zip(w, f)]
    elif kind == "dims":
        at = [rot * math.log(trained / (2.0 * math.pi * n)) / (2.0 * math.log(theta)) for n in (many, few)]
        lo, hi = max(math.floor(at[0]), 0.0), min(math.ceil(at[1]), rot - 1.0)
        w = [1.0 - min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0) for i in range(rot // 2)]
        f = [a * x + (1.0 - a) * x / factor for a, x in zip(w, f)]
        amplitude = 1.0 + 0.1 * math.log(factor)
    t = [int(round(x * 2.0 ** 64)) for x in f]
    return torch.tensor([x - (1 << 64) if x >= 1 << 63 else x for x in t], dtype=torch.int64), amplitude


def _draw_cache(case, g, h, room, most):
    """A cache with room[b] tokens for sequence b, in a pool for `most` tokens of
    every sequence (the rest is what earlier sequences left): K, V
    [page][Hkv][P][dh] with a random page table, or [slots][Hkv][dh]; e4m3 with
    fp32 scales per (token, head)."""
    _, hkv, dh, _ = LAYERS[case["layer"]]
    P = case["page"]
    c = {}
    if P:
        pages = (room + P - 1) // P
        table = torch.full((len(room), (most + P - 1) // P), -1, dtype=torch.int32)
        used = torch.arange(table.shape[1])[None] < pages[:, None]
        total = len(room) * ((most + P - 1) // P)
        table[used] = torch.randperm(total, generator=h)[:int(pages.sum())].to(torch.int32)
        c["table"] = table.cuda()
        shape, at = (total, hkv, P, dh), (total, hkv, P)
    else:
        total = len(room) * most
        c["start"] = (torch.cumsum(room, 0) - room).to(torch.int64).cuda()
        shape, at = (total, hkv, dh), (total, hkv)
    for n in ("k", "v"):
        x = _normal(g, shape)
        x *= torch.exp(0.3 * _normal(g, at))[..., None]
        if case["cache"] == "e4m3":
            amax = x.abs().amax(-1).clamp_min(2.0 ** -60)
            c[n] = (x * (torch.full_like(amax, 448.0) / amax)[..., None]).to(torch.float8_e4m3fn)
            c[n + "_scale"] = amax / 448.0
        else:
            c[n] = x.to(DTYPES[case["cache"]])
        del x
    return c


def _draw_tree(h, B, N, ragged):
    """Random trees: node i hangs on an earlier node (often the one before) or on
    the sequence's last token.  Masks [B][N] (bit j: node j is i or above it),
    node counts [B]; the nodes past a smaller tree's count see nothing."""
    n = _int(h, max(1, N // 2), N, (B,)) if ragged else torch.full((B,), N, dtype=torch.int32)
    up = torch.randint(0, 1 << 30, (B, N), generator=h) % (torch.arange(N)[None] + 1) - 1
    last = torch.rand((B, N), generator=h) < 0.5
    up = torch.where(last, torch.arange(N)[None] - 1, up)
    mask = torch.zeros((B, N), dtype=torch.int64)
    for i in range(N):
        above = mask.gather(1, up[:, i:i + 1].clamp_min(0))[:, 0]
        mask[:, i] = torch.where(up[:, i] >= 0, above, torch.zeros_like(above)) | (-(1 << 63) if i == 63 else 1 << i)
    mask[torch.arange(N)[None] >= n[:, None]] = 0
    return mask, n


def _draw(case, seed):
    g, h = _generators(seed)
    hq, hkv, dh, d = LAYERS[case["layer"]]
    dt = DTYPES[case["dtype"]]
    spread = 0.02 * math.sqrt(d)
    op = case["op"]
    s = {}
    if op == "rotate":
        rot = case["rot"] or dh
        s["x"] = _normal(g, (case["n"], hq + 2 * hkv, dh), spread).to(dt)
        s["pos"] = _int(h, 0, case["far"], (case["n"],)).cuda()
        s["turns"], s["amplitude"] = _turns(case, rot)
        s["turns"] = s["turns"].cuda()
        return s
    B = case["B"]
    lens = _int(h, case["lo"], case["hi"], (B,)).to(torch.int64)
    s["lens"] = lens.to(torch.int32).cuda()
    if op == "append":
        new = _int(h, case["new_lo"], case["new_hi"], (B,)).to(torch.int64)
        s["cache"] = _draw_cache(case, g, h, lens + new, max(case["hi"] + case["new_hi"], 1))
        s["count"] = new.to(torch.int32).cuda()
        s["most"] = max(case["new_hi"], 1)
        if case["take"]:
            total = B * case["take"]
            s["row0"] = (torch.arange(B, dtype=torch.int32) * case["take"]).cuda()
            path = torch.rand((B, case["take"]), generator=h).argsort(1)[:, :s["most"]]
            s["take"] = path.sort(1).values.to(torch.int32).cuda()
        else:
            total = max(int(new.sum()), 1)
            s["row0"] = (torch.cumsum(new, 0) - new).to(torch.int32).cuda()
        s["k"] = _normal(g, (total, hkv, dh), spread).to(dt)
        s["v"] = _normal(g, (total, hkv, dh), spread).to(dt)
        s["turns"], s["amplitude"] = _turns(case, dh)
        s["turns"] = s["turns"].cuda()
        return s
    s["cache"] = _draw_cache(case, g, h, lens, max(case["hi"], 1))
    s["longest"] = max(case["hi"], 1)
    if op == "tree":
        N = case["nodes"]
        s["q"] = _normal(g, (B, N, hq, dh), spread).to(dt)
        s["k_new"] = _normal(g, (B, N, hkv, dh), 1.0).to(dt)
        s["v_new"] = _normal(g, (B, N, hkv, dh), 1.0).to(dt)
        mask, n = _draw_tree(h, B, N, case["ragged"])
        s["mask"], s["n"] = mask.cuda(), n.cuda()
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
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    dt = {"f32": sp.SP_F32, "bf16": sp.SP_BF16, "e4m3": sp.SP_E4M3}
    p = {"sp": sp, "dtype": dt[case["dtype"]]}
    out = DTYPES[case["dtype"]]
    if "turns" in s:
        rot = 2 * s["turns"].numel()
        p["rot"] = sp.sp_rotary(dh, rot, int(case.get("pairs", False)), s["amplitude"], s["turns"].data_ptr())
    if case["op"] == "rotate":
        p["y"] = torch.empty((case["n"], hq + hkv, dh), dtype=out, device="cuda")
        return p
    c, B, P = s["cache"], case["B"], case["page"]
    room = case["hi"] + (case["new_hi"] if case["op"] == "append" else 0)
    if P:
        kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, c["k"].data_ptr(), c["v"].data_ptr(),
                            c["table"].data_ptr(), P, c["k"].shape[0], c["table"].shape[1], B)
        scales = [c[n].data_ptr() if n in c else None for n in ("k_scale", "v_scale")]
    else:
        step = hkv * dh * c["k"].element_size()
        p["at"] = [c[n].data_ptr() + c["start"] * step for n in ("k", "v")]
        kv = sp.sp_kv_cache(sp.SP_KV_CONTIGUOUS, p["at"][0].data_ptr(), p["at"][1].data_ptr(), None, None, None,
                            0, 0, 0, B)
        p["at"] += [c[n].data_ptr() + c["start"] * (hkv * 4) for n in ("k_scale", "v_scale") if n in c]
        scales = [t.data_ptr() for t in p["at"][2:]] or [None, None]
    p["cache"] = sp.sp_token_cache(kv, dt[case["cache"]], hkv, dh, max(room, 1), *scales)
    if case["op"] == "append":
        take = s["take"].data_ptr() if "take" in s else None
        p["rows"] = sp.sp_token_rows(s["row0"].data_ptr(), s["count"].data_ptr(), take, s["most"], s["k"].shape[0], 0, 0)
    elif case["op"] == "read":
        shape = (B, s["longest"], hkv, dh)
        p["k"], p["v"] = (torch.empty(shape, dtype=out, device="cuda") for _ in range(2))
        p["rows"] = sp.sp_token_rows(None, None, None, s["longest"], B * s["longest"], 0, 0)
    else:
        p["dims"] = sp.sp_tree_dims(hq, case["nodes"], p["dtype"], 0, 0, 0.0, 0, 0, 0)
        p["bytes"] = sp.sp_attend_tree_workspace_bytes(p["dims"], p["cache"], B)
        p["ws"] = torch.empty(max(p["bytes"], 1), dtype=torch.uint8, device="cuda")
        p["out"] = torch.empty((B, case["nodes"], hq, dh), dtype=out, device="cuda")
    return p


def prepare(case, seed):
    s = _draw(case, seed)
    s["case"] = case
    if own:
        s["plan"] = _plan(case, s)
    torch.cuda.synchronize()
    return s


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def run(s):
    return _call(s) if own else {"rotate": _plain_rotate, "append": _plain_append, "read": _plain_read,
                                 "tree": _plain_tree}[s["case"]["op"]](s)


def _call(s):
    case, p, st = s["case"], s["plan"], _stream()
    sp, op = p["sp"], case["op"]
    if op == "rotate":
        x, y = s["x"], p["y"]
        sp.sp_rotate(st, p["rot"], case["n"], s["pos"], int(case["backward"]), p["dtype"], y.shape[1], x, x.stride(0),
                     x.stride(1), y, y.stride(0), y.stride(1))
        return y
    if op == "append":
        sp.sp_cache_append(st, p["cache"], p["rot"] if case["rope"] else None, case["B"], None, s["lens"], p["rows"],
                           p["dtype"], s["k"], s["v"])
        return {n: s["cache"][n] for n in ("k", "v", "k_scale", "v_scale") if n in s["cache"]}
    if op == "read":
        sp.sp_cache_read(st, p["cache"], case["B"], None, s["lens"], None, p["rows"], p["dtype"], p["k"], p["v"])
        return [p["k"], p["v"]]
    sp.sp_attend_tree(st, p["dims"], p["cache"], case["B"], None, s["lens"], s["mask"], s["n"], s["q"], s["k_new"],
                      s["v_new"], p["out"], p["ws"], p["bytes"])
    return p["out"]


def _plain_turn(x, pos, turns, amplitude, pairs, backward=False):
    """x [n][heads][dh] (fp32) rotated at pos [n]: the phase p f mod one turn is
    exact in wrapping 64-bit integers, everything else is in 32 bits."""
    r = turns.numel()
    angle = (pos.to(torch.int64)[:, None] * turns[None]).to(torch.float32) * (2.0 * math.pi / 2.0 ** 64)
    c, sn = torch.cos(angle)[:, None] * amplitude, torch.sin(angle)[:, None] * amplitude
    sn = -sn if backward else sn
    if pairs:
        u, v = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        y = torch.stack([u * c - v * sn, v * c + u * sn], dim=-1).flatten(-2)
    else:
        u, v = x[..., :r], x[..., r:2 * r]
        y = torch.cat([u * c - v * sn, v * c + u * sn], dim=-1)
    return torch.cat([y, x[..., 2 * r:]], dim=-1)


def _plain_rotate(s):
    case = s["case"]
    hq, hkv, _, _ = LAYERS[case["layer"]]
    x = s["x"][:, :hq + hkv].to(torch.float32)
    return _plain_turn(x, s["pos"], s["turns"], s["amplitude"], case["pairs"], case["backward"]).to(s["x"].dtype)


def _plain_append(s):
    case, c = s["case"], s["cache"]
    j = torch.arange(s["most"], device="cuda")
    keep = j[None] < s["count"][:, None]
    b, j = keep.nonzero(as_tuple=True)
    row = (s["row0"][b] + (s["take"][b, j] if "take" in s else j)).to(torch.int64)
    t = s["lens"][b].to(torch.int64) + j
    for n in ("k", "v"):
        x = s[n][row].to(torch.float32)
        if n == "k" and case["rope"]:
            x = _plain_turn(x, t, s["turns"], s["amplitude"], False)
        scale = None
        if case["cache"] == "e4m3":
            amax = x.abs().amax(-1).clamp_min(2.0 ** -60)
            # (a scalar over a tensor would be a reciprocal and a product)
            scale, x = amax / 448.0, x * (torch.full_like(amax, 448.0) / amax)[..., None]
        if case["page"]:
            P = case["page"]
            at = (c["table"][b, t // P].to(torch.int64), slice(None), t % P)
        else:
            at = (c["start"][b] + t,)
        # an 8-bit element is written through its bit pattern (indexing has no 8-bit float form)
        dst = c[n].view(torch.uint8) if scale is not None else c[n]
        dst[at] = x.to(c[n].dtype).view(torch.uint8) if scale is not None else x.to(c[n].dtype)
        if scale is not None:
            c[n + "_scale"][at] = scale
    return {n: c[n] for n in ("k", "v", "k_scale", "v_scale") if n in c}


def _plain_gather(s, n):
    """Keys or values [B][longest][Hkv][dh] in fp32, zero past each sequence's end."""
    c, case = s["cache"], s["case"]
    B, T = case["B"], s["longest"]
    x = c[n].view(torch.uint8) if case["cache"] == "e4m3" else c[n]
    scale = c.get(n + "_scale")
    if case["page"]:
        table = c["table"].to(torch.int64).clamp_min(0)
        x = x[table].transpose(2, 3).flatten(1, 2)[:, :T]
        scale = scale[table].transpose(2, 3).flatten(1, 2)[:, :T] if scale is not None else None
    else:
        at = (c["start"][:, None] + torch.arange(T, device="cuda")[None]).clamp_max(x.shape[0] - 1)
        x, scale = x[at], scale[at] if scale is not None else None
    x = (x.view(torch.float8_e4m3fn) if scale is not None else x).to(torch.float32)
    x = x * scale[..., None] if scale is not None else x
    inside = torch.arange(T, device="cuda")[None] < s["lens"][:, None]
    return torch.where(inside[:, :, None, None], x, torch.zeros((), device="cuda"))


def _plain_read(s):
    dt = DTYPES[s["case"]["dtype"]]
    return [_plain_gather(s, "k").to(dt), _plain_gather(s, "v").to(dt)]


def _plain_tree(s):
    case = s["case"]
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    B, N, T, G = case["B"], case["nodes"], s["longest"], hq // hkv
    q = s["q"].to(torch.float32).view(B, N, hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * G, dh)
    alive = torch.arange(N, device="cuda")[None] < s["n"][:, None]
    fresh = [torch.where(alive[:, :, None, None], s[n].to(torch.float32), torch.zeros((), device="cuda"))
             for n in ("k_new", "v_new")]
    k = torch.cat([_plain_gather(s, "k"), fresh[0]], 1).permute(0, 2, 3, 1)
    sees = ((s["mask"][:, :, None] >> torch.arange(N, device="cuda")) & 1).to(torch.bool) & alive[:, :, None] & alive[:, None]
    inside = (torch.arange(T, device="cuda")[None] < s["lens"][:, None])[:, None] & alive[:, :, None]
    sees = torch.cat([inside, sees], 2).repeat_interleave(G, 1)[:, None]
    sc = torch.matmul(q, k) * (1.0 / math.sqrt(dh))
    del k
    sc = sc.masked_fill_(~sees, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp_(sc.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    v = torch.cat([_plain_gather(s, "v"), fresh[1]], 1).permute(0, 2, 1, 3)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(B, hkv, N, G, dh).permute(0, 2, 1, 3, 4).reshape(B, N, hq, dh).to(DTYPES[case["dtype"]])


# --------------------------------------------------------------------------- #
# what a pass cannot do without
# --------------------------------------------------------------------------- #
def work(case):
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    e = BYTES[case["dtype"]]
    if case["op"] == "rotate":
        return {"bytes": case["n"] * ((hq + hkv) * dh * 2.0 * e + 4), "flops": 3.0 * case["n"] * (hq + hkv) * (case["rot"] or dh)}
    token = 2.0 * hkv * (dh * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))  # cached K and V
    cached = case["B"] * (case["lo"] + case["hi"]) / 2.0
    if case["op"] == "append":
        rows = case["B"] * (case["new_lo"] + case["new_hi"]) / 2.0
        return {"bytes": rows * (token + 2.0 * hkv * dh * e) + 12.0 * case["B"], "flops": 6.0 * rows * hkv * dh}
    if case["op"] == "read":
        return {"bytes": cached * token + 2.0 * case["B"] * case["hi"] * hkv * dh * e, "flops": 2.0 * cached * hkv * dh}
    rows = case["B"] * case["nodes"]
    return {"bytes": cached * token + rows * (dh * e * 2.0 * (hq + hkv) + 8), "flops": 4.0 * dh * hq * case["nodes"] * (cached + rows)}


# --------------------------------------------------------------------------- #
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------- #
def _frequencies64(case, rot):
    """Radians a position turns pair i, and the amplitude."""
    kind, factor, trained, few, many = _scaling(case, rot)
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = THETA * factor ** (rot / (rot - 2)) if kind == "base" else THETA
    w = torch.pow(torch.tensor(base, dtype=torch.float64), -2.0 * i / rot)
    if kind == "linear":
        return w / factor, 1.0
    if kind == "turns":
        keep = ((trained * w / (2 * math.pi) - few) / (many - few)).clamp(0, 1)
        return w * (keep + (1 - keep) / factor), 1.0
    if kind == "dims":
        pair = lambda n: rot / 2 * math.log(trained / (n * 2 * math.pi)) / math.log(base)  # noqa: E731
        a, b = max(math.floor(pair(many)), 0), min(math.ceil(pair(few)), rot - 1)
        keep = 1 - ((i - a) / max(b - a, 1e-3)).clamp(0, 1)
        return w * (keep + (1 - keep) / factor), 1 + math.log(factor) / 10
    return w, 1.0


def _turn64(case, x, pos, rot, backward=False):
    w, a = _frequencies64(case, rot)
    z = torch.polar(torch.full((), a, dtype=torch.float64, device=x.device), pos.double()[:, None] * w.to(x.device))[:, None]
    z = z.conj() if backward else z
    y = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case.get("pairs") else (slice(0, rot // 2), slice(rot // 2, rot))
    t = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
    y[..., first], y[..., second] = t.real, t.imag
    return y


def _e4m3_64(x):
    """Nearest value of 1 sign, 4 exponent (bias 7) and 3 mantissa bits, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _cached64(case, s, b, n):
    """Keys or values [L][Hkv][dh] of sequence b."""
    c, L, P = s["cache"], int(s["lens"][b]), case["page"]
    if P:
        pages = c["table"][b, :-(-L // P)].long()
        pick = lambda t: torch.cat([t[int(i)].transpose(0, 1) for i in pages] or [t[0].transpose(0, 1)[:0]])[:L]  # noqa: E731
    else:
        o = int(c["start"][b])
        pick = lambda t: t[o:o + L]  # noqa: E731
    x = pick(c[n].view(torch.uint8)).view(torch.float8_e4m3fn).float().double() if case["cache"] == "e4m3" else pick(c[n]).double()
    return x * pick(c[n + "_scale"]).double()[..., None] if case["cache"] == "e4m3" else x


def exact(case, seed):
    s = _draw(case, seed)
    hq, hkv, dh, _ = LAYERS[case["layer"]]
    if case["op"] == "rotate":
        return _turn64(case, s["x"][:, :hq + hkv].double(), s["pos"], case["rot"] or dh, case["backward"])
    B = case["B"]
    if case["op"] == "append":
        c = s["cache"]
        out = {n: c[n].float().double() if n in ("k", "v") else c[n].double() for n in ("k", "v", "k_scale", "v_scale") if n in c}
        for b in range(B):
            n_new, L, o = int(s["count"][b]), int(s["lens"][b]), int(s["row0"][b])
            rows = o + (s["take"][b, :n_new].long() if "take" in s else torch.arange(n_new, device="cuda"))
            pos = L + torch.arange(n_new, device="cuda")
            for n in ("k", "v"):
                x = s[n][rows].double()
                if n == "k" and case["rope"]:
                    x = _turn64(case, x, pos, dh)
                if case["page"]:
                    at = (c["table"][b].long()[pos // case["page"]], slice(None), pos % case["page"])
                else:
                    at = (int(c["start"][b]) + pos,)
                if case["cache"] == "e4m3":
                    scale = x.abs().amax(-1).clamp_min(2.0 ** -60) / 448.0
                    out[n + "_scale"][at] = scale
                    x = _e4m3_64(x / scale[..., None])
                out[n][at] = x
        return out
    if case["op"] == "read":
        out = [torch.zeros((B, s["longest"], hkv, dh), dtype=torch.float64, device="cuda") for _ in range(2)]
        for b in range(B):
            for o, n in zip(out, ("k", "v")):
                o[b, :int(s["lens"][b])] = _cached64(case, s, b, n)
        return out
    N, G = case["nodes"], hq // hkv
    out = torch.zeros((B, N, hq, dh), dtype=torch.float64, device="cuda")
    bits = torch.arange(64, device="cuda")
    for b in range(B):
        n = int(s["n"][b])
        K, V = (torch.cat([_cached64(case, s, b, c), s[c + "_new"][b, :n].double()]) for c in ("k", "v"))
        sees = torch.ones((n, K.shape[0]), dtype=torch.bool, device="cuda")
        sees[:, K.shape[0] - n:] = ((s["mask"][b, :n, None] >> bits) & 1)[:, :n].bool()
        for g in range(hkv):
            q = s["q"][b, :n, g * G:(g + 1) * G].double().transpose(0, 1)
            sc = (q @ K[:, g].T / math.sqrt(dh)).masked_fill(~sees, -math.inf)
            out[b, :n, g * G:(g + 1) * G] = (torch.softmax(sc, -1).nan_to_num(0.0) @ V[:, g]).transpose(0, 1)
    return out
