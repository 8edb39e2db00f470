"""The decoding loop of examples/tree_decode.py: prompts, trees and accepted paths over one
cache, step by step against float64 attention over what the cache holds, then the probe on it."""
import importlib.util
import os
import types

import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from conftest import ROOT
from gpu_util import ensure_built, torch_dev
from test_gpu_tree import bound
from token_cache_util import quantise, tree_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def load_example():
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
def test_trees_and_accepted_paths_step_by_step(torch, cdt):
    ex = load_example()
    B, hq, hkv, dh, N = 3, 4, 2, 128, 7
    counts = [130, 0, 37]
    dec = ex.TreeDecoder(B, hq, hkv, dh, 260, N, cdt, theta=1.0e4, seed=5)
    g = torch.Generator(device="cuda").manual_seed(3)
    rng = np.random.default_rng(3)

    def rows(n):
        return torch.randn((n, dec.width), generator=g, device="cuda").to(torch.bfloat16)

    dec.prefill(rows(sum(counts)), counts)
    for step in range(3):
        lens = dec.lens.tolist()
        k, v = (x.cpu().double() for x in dec.read())
        held = types.SimpleNamespace(hkv=hkv, values=lambda s, n, which: (k if which == "k" else v)[s, :n])
        trees = [ex.draft(rng, int(rng.integers(1, N + 1))) for _ in range(B)]
        nodes = rows(B * N)
        out = dec.attend(nodes, trees).cpu().double()
        q, kn, vn = (x.cpu().view(B, N, -1, dh) for x in dec._parts(nodes))
        for b, tree in enumerate(trees):
            n, masks = len(tree), sp.sp_tree_masks(tree)[0]
            o, oa, spread = tree_reference(held, b, lens[b], q[b, :n], kn[b, :n], vn[b, :n], masks, dh ** -0.5)
            assert bool(((out[b, :n] - o).abs() <= bound(o, oa, spread, sp.SP_BF16, cdt, True)).all())
            assert bool((out[b, n:] == 0).all())
        paths = [ex.path_to(t, int(rng.integers(0, len(t)))) for t in trees]
        dec.accept(nodes, paths)
        assert dec.lens.tolist() == [n + len(p) for n, p in zip(lens, paths)]
        # what was appended: the accepted nodes' rows, exactly or by the documented codes
        k2, v2 = (x.cpu() for x in dec.read())
        for b, path in enumerate(paths):
            for got, new in ((k2, kn), (v2, vn)):
                want = new[b, path].float()
                if cdt == sp.SP_E4M3:
                    codes, scale = quantise(want)
                    want = codes.float() * scale[..., None]
                at = got[b, lens[b]:lens[b] + len(path)]
                assert bool(((at - want).abs() <= 2.0 ** -22 * want.abs()).all())
            assert bool((k2[b, :lens[b]].double() == k[b, :lens[b]]).all())  # the rest is untouched
    dec.check()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_the_example_runs(torch, cache, monkeypatch, capsys):
    ex = load_example()
    monkeypatch.setattr("sys.argv", ["tree_decode.py", "--cache", cache, "--batch", "3", "--steps", "2"])
    ex.main()
    said = capsys.readouterr().out
    assert "contexts read back" in said and ("probe's classes" in said) == (cache == "bf16")
