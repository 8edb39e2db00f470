"""Host side of the token-cache operators (no GPU): frequency tables against their
definition, tree masks, refusals before any launch, and the kernels' stream order."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from conftest import ROOT
from paper_2608_28099_gb300 import build_lib

INVALID, UNSUPPORTED = sp.SP_ERR_INVALID_ARG, sp.SP_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_lib.build()
    return sp.load_library()


def refused(status, call, *args, text=None):
    with pytest.raises(sp.SpError) as e:
        call(*args)
    assert e.value.status == status, str(e.value)
    if text:
        assert text in str(e.value)


# ---- frequencies -----------------------------------------------------------
def _radians(turns):
    return np.array([int(t) / 2.0 ** 64 * 2 * math.pi for t in turns])


@pytest.mark.parametrize("rot", [2, 4, 32, 64, 128, 130])
@pytest.mark.parametrize("theta", [1.0e4, 5.0e5])
def test_plain_and_linear_frequencies(rot, theta):
    want = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    t, a = sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, rot, theta)
    # 2^-62 turn of rounding, 2^-52 of the double's own
    assert a == 1.0 and np.all(np.abs(_radians(t) - want) <= want * 1e-14 + 2 * math.pi * 2.0 ** -62)
    t, a = sp.sp_rotary_plan(sp.SP_ROPE_LINEAR, rot, theta, 8.0)
    assert a == 1.0 and np.all(np.abs(_radians(t) - want / 8) <= want * 1e-14 + 2 * math.pi * 2.0 ** -62)


def test_stretched_base_keeps_the_fastest_pair_and_divides_the_slowest():
    t0, _ = sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, 64)
    t1, _ = sp.sp_rotary_plan(sp.SP_ROPE_BASE, 64, factor=4.0)
    r = _radians(t1) / _radians(t0)
    assert abs(r[0] - 1) < 1e-14 and abs(r[-1] - 0.25) < 1e-12 and np.all(np.diff(r) < 0)


def test_ramps_by_turns_and_by_dims():
    L0, s = 8192.0, 8.0
    f = _radians(sp.sp_rotary_plan(sp.SP_ROPE_PLAIN, 128)[0])
    turns = L0 * f / (2 * math.pi)
    t, a = sp.sp_rotary_plan(sp.SP_ROPE_TURNS, 128, factor=s, trained_len=L0, few=1.0, many=4.0)
    r = _radians(t) / f
    assert a == 1.0
    assert np.allclose(r[turns >= 4], 1, atol=1e-12) and np.allclose(r[turns <= 1], 1 / s, atol=1e-12)
    mid = (turns > 1) & (turns < 4)
    w = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(r[mid], w + (1 - w) / s, atol=1e-12)
    t, a = sp.sp_rotary_plan(sp.SP_ROPE_DIMS, 128, factor=s, trained_len=L0, few=1.0, many=32.0)
    r = _radians(t) / f
    assert abs(a - (1 + 0.1 * math.log(s))) < 1e-6
    kept, divided = np.isclose(r, 1, atol=1e-9), np.isclose(r, 1 / s, atol=1e-9)
    assert np.all(kept[turns > 40]) and np.all(divided[turns < 0.8]) and np.all(np.diff(r) <= 1e-12)
    steps = np.diff(r[~kept & ~divided])  # linear in the pair index
    assert len(steps) > 3 and np.allclose(steps, steps[0], atol=1e-9)


@pytest.mark.parametrize("args", [
    (9, 64, 1e4, 1.0, 0, 1, 2), (-1, 64, 1e4, 1.0, 0, 1, 2), (0, 63, 1e4, 1.0, 0, 1, 2), (0, 0, 1e4, 1.0, 0, 1, 2),
    (0, 2048, 1e4, 1.0, 0, 1, 2), (0, 64, 1.0, 1.0, 0, 1, 2), (0, 64, float("nan"), 1.0, 0, 1, 2),
    (1, 64, 1e4, 0.5, 0, 1, 2), (2, 2, 1e4, 2.0, 0, 1, 2), (3, 64, 1e4, 2.0, 0, 1, 2), (3, 64, 1e4, 2.0, 100, 2, 2),
    (4, 64, 1e4, 2.0, 100, 0, 2), (4, 64, 1e4, 2.0, 100, 1, float("inf"))])
def test_bad_frequency_plans_are_refused(args):
    refused(INVALID, sp.sp_rotary_plan, *args)


# ---- trees -----------------------------------------------------------------
def test_masks_and_depths_of_a_tree():
    masks, depths = sp.sp_tree_masks([-1, 0, 0, 1, -1, 4, 3])
    assert [int(m) for m in masks] == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b110000, 0b1001011]
    assert list(depths) == [0, 1, 1, 2, 0, 1, 3]
    masks, depths = sp.sp_tree_masks(list(range(-1, 63)))
    assert int(masks[63]) == 2 ** 64 - 1 and depths[63] == 63


@pytest.mark.parametrize("parents", [[0], [-2], [-1, 1], [-1, 0, 5], []])
def test_bad_trees_are_refused(parents):
    refused(INVALID, sp.sp_tree_masks, parents)


def test_a_tree_of_65_nodes_is_refused():
    refused(INVALID, sp.sp_tree_masks, list(range(-1, 64)))


# ---- refusals (the fake addresses are never dereferenced) -------------------
def _rot(**over):
    r = dict(head_dim=128, rot_dim=128, interleaved=0, amplitude=1.0, d_turns=0x1000)
    r.update(over)
    return sp.sp_rotary(*r.values())


def _rotate(rot=None, **over):
    a = dict(n=4, pos=0x2000, backward=0, dtype=sp.SP_BF16, heads=2, x=0x10000, xt=256, xh=128, y=0x20000, yt=256, yh=128)
    a.update(over)
    sp.sp_rotate(None, rot or _rot(), *a.values())


@pytest.mark.parametrize("over", [
    dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=130), dict(head_dim=0), dict(head_dim=2000), dict(interleaved=2),
    dict(amplitude=float("nan")), dict(d_turns=None)])
def test_bad_rotaries_are_refused(over):
    refused(INVALID, _rotate, _rot(**over))


@pytest.mark.parametrize("over", [
    dict(n=-1), dict(pos=None), dict(backward=2), dict(dtype=sp.SP_E4M3), dict(heads=0), dict(x=None), dict(y=None),
    dict(x=0x10001), dict(yt=-1), dict(yh=64), dict(yt=100), dict(y=0x10000, yt=512)])
def test_bad_rotations_are_refused(over):
    refused(INVALID, lambda: _rotate(**over))


def _kv(**over):
    k = dict(layout=sp.SP_KV_PAGED, k_seq=None, v_seq=None, k_pool=0x100000, v_pool=0x200000, page_table=0x300000,
             page_size=16, n_pages=8, max_pages_per_seq=4, n_seqs=4)
    k.update(over)
    return sp.sp_kv_cache(*k.values())


def _cache(kv=None, **over):
    c = dict(dtype=sp.SP_E4M3, hkv=2, dh=128, max_len=64, ks=0x400000, vs=0x500000)
    c.update(over)
    return sp.sp_token_cache(kv or _kv(), *c.values())


def _rows(**over):
    r = dict(row0=None, count=None, take=None, max_rows=4, n_rows=16, ks=0, vs=0)
    r.update(over)
    return sp.sp_token_rows(*r.values())


def _append(cache=None, rows=None, rot=None, batch=4, lens=0x600000, dtype=sp.SP_BF16, k=0x700000, v=0x800000):
    sp.sp_cache_append(None, cache or _cache(), rot, batch, None, lens, rows or _rows(), dtype, k, v)


def _read(cache=None, rows=None, batch=4, lens=0x600000, dtype=sp.SP_BF16, k=0x700000, v=0x800000):
    sp.sp_cache_read(None, cache or _cache(), batch, None, lens, None, rows or _rows(), dtype, k, v)


BAD_CACHES = [
    (INVALID, lambda: _cache(dtype=3)), (INVALID, lambda: _cache(hkv=0)), (UNSUPPORTED, lambda: _cache(dh=96)),
    (INVALID, lambda: _cache(max_len=-1)), (INVALID, lambda: _cache(ks=None)), (INVALID, lambda: _cache(vs=0x500004)),
    (INVALID, lambda: _cache(_kv(n_seqs=0))), (INVALID, lambda: _cache(_kv(layout=5))),
    (INVALID, lambda: _cache(_kv(k_pool=0x100008))), (UNSUPPORTED, lambda: _cache(_kv(page_size=24))),
    (INVALID, lambda: _cache(_kv(n_pages=0))), (INVALID, lambda: _cache(_kv(page_table=None))),
    (INVALID, lambda: _cache(_kv(layout=sp.SP_KV_CONTIGUOUS)))]


@pytest.mark.parametrize("i", range(len(BAD_CACHES)))
def test_bad_caches_are_refused(i):
    status, make = BAD_CACHES[i]
    refused(status, _append, make())
    refused(status, _read, make())
    refused(status, _tree, make())


@pytest.mark.parametrize("call", [_append, _read])
@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(batch=5), dict(lens=None), dict(dtype=sp.SP_E4M3), dict(k=None), dict(v=None), dict(k=0x700001),
    dict(rows=dict(max_rows=0)), dict(rows=dict(n_rows=0)), dict(rows=dict(ks=255)), dict(rows=dict(vs=100))])
def test_bad_copies_are_refused(call, kw):
    kw = dict(kw)
    if "rows" in kw:
        kw["rows"] = _rows(**kw["rows"])
    refused(INVALID, lambda: call(**kw))


def test_an_append_with_another_head_dim_in_its_rotary_is_refused():
    refused(INVALID, lambda: _append(rot=_rot(head_dim=64, rot_dim=64)), text="head_dim")


def _dims(**over):
    d = dict(hq=8, nodes=8, dtype=sp.SP_BF16, path=0, shared=0, scale=0.0, qs=0, ks=0, vs=0)
    d.update(over)
    return sp.sp_tree_dims(*d.values())


def _tree(cache=None, dims=None, batch=4, **over):
    a = dict(lens=0x600000, mask=None, n=None, q=0x700000, k=0x800000, v=0x900000, out=0xA00000, ws=0xB00000, size=1 << 40)
    a.update(over)
    sp.sp_attend_tree(None, dims or _dims(), cache or _cache(), batch, None, *a.values())


@pytest.mark.parametrize("over", [
    dict(hq=0), dict(hq=3), dict(nodes=0), dict(nodes=65), dict(dtype=sp.SP_E4M3), dict(path=3), dict(path=-1),
    dict(shared=2), dict(scale=-1.0), dict(scale=float("inf")), dict(qs=100), dict(ks=8), dict(qs=1028), dict(vs=260)])
def test_bad_tree_dims_are_refused(over):
    refused(INVALID, lambda: _tree(dims=_dims(**over)))
    assert sp.sp_attend_tree_workspace_bytes(_dims(**over), _cache(), 4) == 0


@pytest.mark.parametrize("over", [
    dict(lens=None), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(ws=None), dict(ws=0xB00010),
    dict(size=16), dict(q=0x700008), dict(k=0x800004), dict(v=0x900002), dict(out=0xA00008), dict(batch=0), dict(batch=5)])
def test_bad_tree_calls_are_refused(over):
    refused(INVALID, lambda: _tree(**over))


def test_the_tensor_path_is_refused_where_it_does_not_apply():
    for dims, cache in [(_dims(path=2, dtype=sp.SP_F32), _cache()), (_dims(path=2), _cache(dh=64)),
                        (_dims(path=2), _cache(dtype=sp.SP_F32, ks=None, vs=None))]:
        refused(UNSUPPORTED, lambda: _tree(dims=dims, cache=cache))


def test_structures_match_the_header():
    """Field names, order and kinds of the new structures."""
    text = open(os.path.join(ROOT, "include", "sp.h")).read()
    text = re.sub(r"/\*.*?\*/", " ", text, flags=re.S)
    for cls in (sp.sp_rotary, sp.sp_token_cache, sp.sp_token_rows, sp.sp_tree_dims):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cls.__name__, cls.__name__), text, re.S).group(1)
        want = []
        for line in [x.strip() for x in body.split(";") if x.strip()]:
            names = re.findall(r"[\s\*](\w+)\s*(?=,|$)", line)
            ptr = "*" in line
            kind = (C.c_void_p if ptr else sp.sp_kv_cache if "sp_kv_cache" in line else C.c_longlong if "long long" in line
                    else C.c_float if line.startswith("float") else C.c_int)
            want += [(n, kind) for n in names]
        assert [(n, t) for n, t in cls._fields_] == want


@pytest.mark.parametrize("name,value", [("SP_ROPE_PLAIN", 0), ("SP_ROPE_LINEAR", 1), ("SP_ROPE_BASE", 2),
                                        ("SP_ROPE_TURNS", 3), ("SP_ROPE_DIMS", 4), ("SP_E4M3", 2), ("SP_DEV_BAD_ROW", 16)])
def test_constants(name, value):
    assert getattr(sp, name) == value


# ---- stream order ------------------------------------------------------------
FIRST = ["rotate_kernel", "append_kernel", "read_kernel", "tree_simt_kernel", "tree_tc_kernel"]


@pytest.mark.parametrize("name", FIRST)
def test_a_first_kernel_touches_the_callers_data_after_its_wait(name):
    from test_launch_order import KERNELS
    body = KERNELS[name]
    before = body[:body.index("pdl_wait()")]
    assert body.index("pdl_wait()") < body.index("pdl_trigger()")
    assert not re.search(r"resolve_seq|tree_nodes|tree_mask|load|a\.pos\[|chunk_of|prefix\(", before)
