"""Queries and keys of drafted nodes near the ends of the range, over 8-bit caches: their two 8-bit
parts are scaled by powers of two, whatever the magnitude."""
import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_tree_nonfinite import DH, HKV, ROWS, Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("power", [60, 119, 121, 124, 126])
def test_node_keys_of_any_magnitude(torch, G, N, power):
    # keys times 2^power, queries times 2^-100, the scale times 2^(100 - power): powers of two
    # change no rounding
    scale = float(np.float32(DH ** -0.5))
    c = Call(torch, sp.SP_E4M3, 2, G, N, [0], scale=scale)
    c.k = c.k.clamp(-1.9, 1.9)
    plain = c.run()
    c.k, c.q, c.dims.scale = c.k * 2.0 ** power, c.q * 2.0 ** -100, scale * 2.0 ** (100 - power)
    assert bool(torch.isfinite(c.k).all())
    assert torch.equal(c.run(), plain)


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("power", [60, 118, 121, 124])
def test_large_queries_find_the_largest_score(torch, path, G, N, power):
    # scores of some 2^(power - 13): one token has all the weight.  (The keys' largest element meets
    # a query of 0, so that the sums of products of codes fit fp32 beside the queries' scale.)
    # Nodes see the cache alone: their own keys are exact to 2^-18 of the largest element only.
    c = Call(torch, sp.SP_E4M3, path, G, N, [200], mask=[0] * N)
    c.q = (c.q.float().clamp(-1.9, 1.9) * 2.0 ** power).to(torch.bfloat16)
    c.kv = [[k * 2.0 ** -13, v] for k, v in c.kv]
    c.q[..., 127], c.kv[0][0][..., 127] = 0.0, 1.0
    out = c.run().double()
    keys, vals = c.cache.values(0, 200, "k"), c.cache.values(0, 200, "v")
    told = 0
    for i in range(N):
        for h in range(HKV * G):
            score = keys[:, h // G] @ c.q[0, i, h].double()
            top = score.sort().values[-2:]
            if float(top[1] - top[0]) < 1e-3 * float(score.abs().max()):
                continue  # a near tie
            told += 1
            want = vals[int(score.argmax()), h // G]
            assert bool(((out[0, i, h] - want).abs() <= 2.0 ** -7 * want.abs()).all())
    assert told > N
