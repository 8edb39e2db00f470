"""Calls of the row norms, the vocabulary loss and the attention's backward pass that are refused, on
the host (no GPU).  They run in a process that sees no device: one that was not refused must not reach
a GPU with the addresses made up here."""
import json
import os
import subprocess
import sys

import pytest

import paper_2608_28099_gb300 as sp
from conftest import ROOT
from paper_2608_28099_gb300 import build_lib

BAD, NOT = sp.SP_ERR_INVALID_ARG, sp.SP_ERR_UNSUPPORTED
P = [0x10000 * (i + 1) for i in range(20)]  # made-up, aligned device addresses
BIG = 1 << 60


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_lib.build()


PROGRAM = """
import json, sys
sys.path.insert(0, {root!r})
import paper_2608_28099_gb300 as sp
def status(name, args):
    args = [getattr(sp, a[0])(*a[1]) if isinstance(a, list) else a for a in args]
    for i, a in enumerate(args):
        if isinstance(a, sp.sp_token_cache):
            pass
    try:
        r = getattr(sp, name)(*args)
        return r if r is not None else 0
    except sp.SpError as e:
        return e.status
def cache(dtype, hkv, dh, page, layout):
    kv = sp.sp_kv_cache(layout, 0x10000, 0x20000, 0x100000, 0x200000, 0x300000, page, 8, 4, 4)
    return sp.sp_token_cache(kv, dtype, hkv, dh, 64, 0x400000, 0x500000)
sp.cache = cache
print(json.dumps([status(n, a) for n, a in json.loads(sys.stdin.read())]))
"""


def answers(calls):
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(root=ROOT)], input=json.dumps(calls), capture_output=True,
                       text=True, timeout=120, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
    assert r.returncode == 0, r.stderr[-800:]
    return json.loads(r.stdout)


def norm_dims(n=4, d=64, dtype=sp.SP_BF16, out=sp.SP_BF16, eps=1e-6, x=0, r=0, s=0, y=0):
    return ["sp_norm_dims", [n, d, dtype, out, eps, x, r, s, y]]


def vocab_dims(n=4, V=50, d=64, dtype=sp.SP_BF16, path=0, h=0, w=0):
    return ["sp_vocab_dims", [n, V, d, dtype, path, h, w]]


def test_norm():
    x, r, g, s, y, sc = P[:6]
    call = lambda dims, *a: ["sp_norm", [None, dims, *a]]  # noqa: E731
    bad = [norm_dims(n=-1), norm_dims(d=0), norm_dims(dtype=sp.SP_E4M3), norm_dims(dtype=7), norm_dims(out=sp.SP_F32),
           norm_dims(eps=-1.0), norm_dims(x=63), norm_dims(r=1), norm_dims(s=-64), norm_dims(y=10)]
    calls = [call(d, x, r, g, s, y, sc) for d in bad]
    calls += [call(norm_dims(), None, r, g, s, y, sc), call(norm_dims(), x, r, g, s, None, sc),
              call(norm_dims(out=sp.SP_E4M3), x, r, g, s, y, None), call(norm_dims(), x + 1, r, g, s, y, sc),
              call(norm_dims(), x, r + 1, g, s, y, sc), call(norm_dims(), x, r, g + 2, s, y, sc),
              call(norm_dims(), x, r, g, s, s, sc), call(norm_dims(out=sp.SP_E4M3), x, r, g, s, x, sc),
              call(norm_dims(x=64, y=72), x, r, g, s, x, sc), call(norm_dims(r=80), x, r, g, r, y, sc),
              call(norm_dims(s=72), x, r, g, x, y, sc), call(norm_dims(dtype=sp.SP_F32, out=sp.SP_F32), x + 2, r, g, s, y, sc)]
    assert answers(calls) == [BAD] * len(calls)
    assert answers([call(norm_dims(d=(1 << 24) + 1), x, r, g, s, y, sc)]) == [NOT]
    assert answers([call(norm_dims(n=0), None, None, None, None, None, None)]) == [0]


def test_norm_backward():
    dy, s, g, ds, dx, dg, ws = P[:7]
    call = lambda dims, *a: ["sp_norm_backward", [None, dims, *a]]  # noqa: E731
    calls = [call(norm_dims(n=-1), dy, s, g, ds, dx, dg, ws, BIG), call(norm_dims(), None, s, g, ds, dx, dg, ws, BIG),
             call(norm_dims(), dy, None, g, ds, dx, dg, ws, BIG), call(norm_dims(), dy, s, g, ds, None, dg, ws, BIG),
             call(norm_dims(), dy, s, g, ds, dx, dg, None, BIG), call(norm_dims(), dy, s, g, ds, dx, dg, ws + 16, BIG),
             call(norm_dims(), dy, s, g, ds, dx, dg, ws, 16), call(norm_dims(), dy + 1, s, g, ds, dx, dg, ws, BIG),
             call(norm_dims(), dy, s, g, ds, dx, dg + 2, ws, BIG), call(norm_dims(x=64, y=72), dy, s, g, ds, dy, dg, ws, BIG),
             call(norm_dims(x=72), dy, s, g, ds, ds, dg, ws, BIG), call(norm_dims(eps=-1e-9), dy, s, g, ds, dx, dg, ws, BIG)]
    assert answers(calls) == [BAD] * len(calls)
    sizes = answers([["sp_norm_backward_workspace_bytes", [d]] for d in (norm_dims(), norm_dims(n=0), norm_dims(d=0))])
    assert sizes[0] > 0 and sizes[1] > 0 and sizes[2] == 0
    assert answers([call(norm_dims(n=0), None, None, None, None, None, None, None, 0)]) == [0]


def test_vocab_loss():
    h, w, t, loss, lse, ws = P[:6]
    call = lambda dims, *a: ["sp_vocab_loss", [None, dims, *a]]  # noqa: E731
    bad = [vocab_dims(n=-1), vocab_dims(V=0), vocab_dims(d=0), vocab_dims(dtype=sp.SP_E4M3), vocab_dims(path=3),
           vocab_dims(path=-1), vocab_dims(h=63), vocab_dims(w=8)]
    calls = [call(d, h, w, t, loss, lse, ws, BIG) for d in bad]
    calls += [call(vocab_dims(), *[None if i == j else p for j, p in enumerate((h, w, t, loss, lse, ws))], BIG) for i in range(6)]
    calls += [call(vocab_dims(), h + 8, w, t, loss, lse, ws, BIG), call(vocab_dims(), h, w + 2, t, loss, lse, ws, BIG),
              call(vocab_dims(dtype=sp.SP_F32), h + 2, w, t, loss, lse, ws, BIG), call(vocab_dims(), h, w, t, loss, lse, ws + 128, BIG),
              call(vocab_dims(), h, w, t, loss, lse, ws, 256),
              call(vocab_dims(), h, w, t + 2, loss, lse, ws, BIG), call(vocab_dims(), h, w, t, loss + 1, lse, ws, BIG),
              call(vocab_dims(), h, w, t, loss, lse + 2, ws, BIG)]
    assert answers(calls) == [BAD] * len(calls)
    refused = [vocab_dims(n=4000001), vocab_dims(V=(1 << 24) + 1), vocab_dims(d=(1 << 20) + 8), vocab_dims(path=2, d=60),
               vocab_dims(path=2, h=68), vocab_dims(path=2, w=68), vocab_dims(path=2, dtype=sp.SP_F32)]
    assert answers([call(d, h, w, t, loss, lse, ws, BIG) for d in refused]) == [NOT] * len(refused)
    assert answers([["sp_vocab_loss_workspace_bytes", [d]] for d in refused + bad]) == [0] * (len(refused) + len(bad))
    assert answers([call(vocab_dims(n=0), None, None, None, None, None, None, 0)]) == [0]


def test_vocab_loss_backward():
    h, w, t, lse, gl, dh, dw, ws = P[:8]
    call = lambda dims, *a: ["sp_vocab_loss_backward", [None, dims, *a]]  # noqa: E731
    args = (h, w, t, lse, gl, dh, dw, ws)
    calls = [call(vocab_dims(), *[None if i == j else p for j, p in enumerate(args)], BIG) for i in (0, 1, 2, 3, 5, 7)]
    calls += [call(vocab_dims(), *[p + 4 if i == j else p for j, p in enumerate(args)], BIG) for i in (0, 1, 5, 6, 7)]
    calls += [call(vocab_dims(), *[p + 2 if i == j else p for j, p in enumerate(args)], BIG) for i in (2, 3, 4)]
    calls += [call(vocab_dims(), *args, 256), call(vocab_dims(d=0), *args, BIG)]
    assert answers(calls) == [BAD] * len(calls)


@pytest.mark.parametrize("n,V,d", [(4000000, 1 << 24, 8), (4000000, 300, 1 << 20), (1, 1 << 24, 1 << 20), (1, 1, 1)])
@pytest.mark.parametrize("dtype,path", [(sp.SP_F32, 0), (sp.SP_BF16, 0), (sp.SP_BF16, 1)])
def test_workspaces_of_the_largest_sizes(n, V, d, dtype, path):
    a, b = answers([["sp_vocab_loss_workspace_bytes", [vocab_dims(n, V, d, dtype, path)]],
                    ["sp_vocab_loss_backward_workspace_bytes", [vocab_dims(n, V, d, dtype, path)]]])
    # at least the kept rows and a piece's gradients, less than that with sixteen copies of dh and tiles' remainders
    assert n * d <= a < 64 * (n + 256) * (V // 64 + d + 64) and n * d <= b < 64 * (n + 100000) * (d + 256) * 4 + (1 << 32)


def tree_dims(hq=4, N=5, dtype=sp.SP_BF16, path=0, shared=0, scale=0.0, q=0, k=0, v=0):
    return ["sp_tree_dims", [hq, N, dtype, path, shared, scale, q, k, v]]


def tree_cache(dtype=sp.SP_BF16, hkv=2, dh=128, page=16, layout=sp.SP_KV_PAGED):
    return ["cache", [dtype, hkv, dh, page, layout]]


def test_attention_backward():
    names = ["lens", "mask", "n", "q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "ws"]
    at = dict(zip(names, P))

    def call(dims=None, cache=None, batch=4, size=BIG, **change):
        a = [{**at, **change}[x] for x in names]
        return ["sp_attend_tree_backward", [None, dims or tree_dims(), cache or tree_cache(), batch, None, *a, size]]
    calls = [call(**{x: None}) for x in names if x not in ("mask", "n")]
    calls += [call(**{x: at[x] + 8}) for x in ("q", "k", "v", "out", "dout", "dq", "dk", "dv", "ws")] + [call(lse=at["lse"] + 2)]
    calls += [call(size=256), call(batch=0), call(batch=5), call(tree_dims(hq=3)), call(tree_dims(N=0)), call(tree_dims(N=65)),
              call(tree_dims(dtype=sp.SP_E4M3)), call(tree_dims(path=3)), call(tree_dims(shared=2)), call(tree_dims(scale=-1.0)),
              call(tree_dims(q=100)), call(tree_dims(k=259)), call(cache=tree_cache(dtype=5))]
    assert answers(calls) == [BAD] * len(calls)
    refused = [call(tree_dims(path=2, dtype=sp.SP_F32)), call(tree_dims(path=2, dtype=sp.SP_F32), tree_cache(sp.SP_E4M3)),
               call(tree_dims(path=2), tree_cache(sp.SP_F32)), call(tree_dims(path=2), tree_cache(dh=64)),
               call(cache=tree_cache(dh=96)), call(cache=tree_cache(page=8)), call(batch=70000)]
    assert answers(refused) == [NOT] * len(refused)


def test_attention_with_log_sums():
    a = P[:10]
    call = lambda lse: ["sp_attend_tree_lse", [None, tree_dims(), tree_cache(), 4, None, a[0], a[1], a[2], a[3], a[4], a[5],  # noqa: E731
                                               a[6], lse, a[7], BIG]]
    assert answers([call(None), call(a[8] + 1)]) == [BAD, BAD]
