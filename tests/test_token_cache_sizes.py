"""Sizes whose products pass 32 bits are refused on the host (no GPU).  The calls run in a
process of their own, without a device: a division by a product that wrapped to 0 would end it,
and a call that is not refused must not reach a GPU with the addresses made up here."""
import os
import subprocess
import sys

import pytest

import paper_2608_28099_gb300 as sp
from conftest import ROOT
from paper_2608_28099_gb300 import build_lib


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_lib.build()


CALLS = """
import sys
sys.path.insert(0, {root!r})
import paper_2608_28099_gb300 as sp
kv = sp.sp_kv_cache({layout}, 0xA0000, 0xB0000, 0x100000, 0x200000, 0x300000, 16, 8, 4, 4)
cache = sp.sp_token_cache(kv, {cache}, {hkv}, {dh}, 64, 0x400000, 0x500000)
def status(call, *args):
    try:
        call(*args)
    except sp.SpError as e:
        return e.status
dims = sp.sp_tree_dims({hq}, {nodes}, {dtype}, {path}, 0, 0.0, 0, 0, 0)
rows = sp.sp_token_rows(None, None, None, 4, 16, 0, 0)
print(sp.sp_attend_tree_workspace_bytes(dims, cache, 4),
      status(sp.sp_attend_tree, None, dims, cache, 4, None, 0x600000, None, None, 0x700000, 0x800000, 0x900000, 0xA00000,
             0xB00000, 1 << 60))
if {copies}:
    print(status(sp.sp_cache_append, None, cache, None, 4, None, 0x600000, rows, 1, 0x700000, 0x800000),
          status(sp.sp_cache_read, None, cache, 4, None, 0x600000, None, rows, 1, 0x700000, 0x800000))
"""


def answers(**kw):
    a = dict(root=ROOT, layout=sp.SP_KV_PAGED, cache=sp.SP_E4M3, hkv=1, dh=128, hq=4, nodes=4, dtype=sp.SP_BF16, path=0,
             copies=False)
    a.update(kw)
    r = subprocess.run([sys.executable, "-c", CALLS.format(**a)], capture_output=True, text=True, timeout=120,
                       env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    return r.stdout.split()


@pytest.mark.parametrize("path", [0, 1, 2])
@pytest.mark.parametrize("hq,nodes", [(1 << 26, 64), (1 << 25, 64), (1 << 30, 4), (1 << 30, 1), ((1 << 26) + 1, 64),
                                      (3 << 25, 64), (2 ** 31 - 1, 64)])
def test_query_rows_past_32_bits(path, hq, nodes):
    got = answers(hq=hq, nodes=nodes, path=path)
    assert got[0] == "0" and int(got[1]) == sp.SP_ERR_UNSUPPORTED


@pytest.mark.parametrize("layout", [sp.SP_KV_PAGED, sp.SP_KV_CONTIGUOUS])
@pytest.mark.parametrize("hkv,dh", [(1 << 27, 32), (1 << 24, 128), (1 << 30, 64), (2 ** 31 - 1, 128)])
def test_heads_past_32_bits(layout, hkv, dh):
    # a block's rows (16 tokens of K and V), and a head's place in a row, are 32-bit numbers
    got = answers(layout=layout, hkv=hkv, dh=dh, hq=hkv, nodes=1, copies=True)
    assert got[0] == "0" and [int(x) for x in got[1:]] == [sp.SP_ERR_UNSUPPORTED] * 3


@pytest.mark.parametrize("batch,hq,hkv,nodes", [(1, 4, 2, 5), (1, 8, 1, 64), (3, 4, 2, 5), (200, 4, 2, 5), (600, 16, 8, 64)])
@pytest.mark.parametrize("longest", [2 ** 30, 2 ** 31 - 5000, 2 ** 31 - 1 - 4096])
def test_the_workspace_of_any_length_bound(batch, hq, hkv, nodes, longest):
    # far above the number of shares the bound changes their length, not their number
    def size(most):
        kv = sp.sp_kv_cache(sp.SP_KV_PAGED, None, None, 0x100000, 0x200000, 0x300000, 16, 8, 4, batch)
        cache = sp.sp_token_cache(kv, sp.SP_F32, hkv, 128, most, None, None)
        return sp.sp_attend_tree_workspace_bytes(sp.sp_tree_dims(hq, nodes, sp.SP_F32, 0, 0, 0.0, 0, 0, 0), cache, batch)
    assert 0 < size(longest) == size(2 ** 26)
