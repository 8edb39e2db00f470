"""NaN and infinities among the values that a row sees, whatever their weight."""
import pytest

import paper_2608_28099_gb300 as sp
from gpu_util import ensure_built, torch_dev
from test_gpu_tree_nonfinite import KINDS, ROWS, Call, same_elsewhere

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def torch():
    ensure_built()
    return torch_dev()


def the_same_kind(torch, got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0.0, 1.0, -1.0), want.nan_to_num(0.0, 1.0, -1.0))


def check_cached_values(torch, cdt, path, G, N, length, scale, pairs):
    """pairs: (token, value) put into dim 7 of head 0; the rows get their sum there (NaN from
    an 8-bit cache, which holds no infinities)."""
    c = Call(torch, cdt, path, G, N, [length, 20], scale=scale)
    for t, _ in pairs:
        c.kv[0][1][t, 0, 7] = 0.0  # (not the element that sets an 8-bit row's scale)
    clean = c.run()
    for t, x in pairs:
        c.kv[0][1][t, 0, 7] = x
    got = c.run()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[0, :, c.heads(0), 7] = True
    the_same_kind(torch, got[touched], torch.full_like(got[touched], sum(x for _, x in pairs) if cdt == sp.SP_BF16 else NAN))
    same_elsewhere(torch, got, clean, touched)


def check_node_values(torch, cdt, path, G, N, length, scale, value):
    """Node 1's value is not finite; it is seen by itself and by nodes 2 and up, beside the cache."""
    c = Call(torch, cdt, path, G, N, [length, 20], scale=scale)
    clean = c.run()
    c.v[:, 1, 0, 7] = value
    got = c.run()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[:, 1:, c.heads(0), 7] = True
    the_same_kind(torch, got[touched], torch.full_like(got[touched], value))
    same_elsewhere(torch, got, clean, touched)


# scores spread over hundreds of powers of two: almost every weight is below 2^-149
STEEP = 40.0


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("length,tokens", [(300, (0, 150, 299)), (2000, (1000,))])
def test_values_of_vanishing_weight_on_cuda_cores(torch, cdt, G, N, value, length, tokens):
    for t in tokens:
        check_cached_values(torch, cdt, 1, G, N, length, STEEP, [(t, value)])
    check_node_values(torch, cdt, 1, G, N, length, STEEP, value)


@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("length,tokens", [(300, (0, 150, 299)), (2000, (1000,))])
def test_values_of_vanishing_weight_from_an_8_bit_cache(torch, G, N, length, tokens):
    for t in tokens:
        check_cached_values(torch, sp.SP_E4M3, 2, G, N, length, STEEP, [(t, NAN)])


@pytest.mark.parametrize("cdt", [sp.SP_BF16, sp.SP_E4M3])
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("length", [40, 300, 2000])
def test_node_values_of_vanishing_weight(torch, cdt, G, N, value, length):
    check_node_values(torch, cdt, 2, G, N, length, STEEP, value)


@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("length,tokens", [(300, (0, 150, 299)), (2000, (1000,))])
def test_values_of_vanishing_weight_from_a_bf16_cache(torch, G, N, value, length, tokens):
    for t in tokens:
        check_cached_values(torch, sp.SP_BF16, 2, G, N, length, STEEP, [(t, value)])


@pytest.mark.parametrize("cdt,path", KINDS)
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("length", [1, 33, 128, 300, 3000])
def test_non_finite_cached_values(torch, cdt, path, G, N, length):
    for pairs in ([(length - 1, INF)], [(0, -INF)], [(length // 2, NAN)]):
        check_cached_values(torch, cdt, path, G, N, length, 0.0, pairs)
    if length > 1:
        for last in (INF, -INF):
            check_cached_values(torch, cdt, path, G, N, length, 0.0, [(0, INF), (length - 1, last)])


@pytest.mark.parametrize("page", [0, 32, 64])
@pytest.mark.parametrize("G,N", ROWS)
def test_infinite_values_in_every_dim_and_layout(torch, page, G, N):
    # every third dim of head 1 infinite somewhere in the context, and the same call once more without
    c = Call(torch, sp.SP_BF16, 2, G, N, [700, 20, 150], page)
    clean = c.run()
    keep = [[k.clone(), v.clone()] for k, v in c.kv]
    touched = torch.zeros_like(clean, dtype=torch.bool)
    want = clean.clone()
    for b in (0, 2):
        for d in range(0, 128, 3):
            value = INF if d % 2 else -INF
            c.kv[b][1][(d * 37) % c.lens[b], 1, d] = value
            touched[b, :, c.heads(1), d] = True
            want[b, :, c.heads(1), d] = value
    got = c.run()
    the_same_kind(torch, got[touched], want[touched])
    same_elsewhere(torch, got, clean, touched)
    c.kv = keep
    assert torch.equal(c.run(), clean)


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("G,N", ROWS)
@pytest.mark.parametrize("length", [40, 900])
def test_cached_and_new_values_meet(torch, path, G, N, length):
    # node 1's value is -inf, a cached one +inf: NaN where a row sees both
    masks = [1 << i | (2 if i > 2 else 0) for i in range(N)]
    c = Call(torch, sp.SP_BF16, path, G, N, [length, 20], mask=masks)
    c.kv[0][1][length - 1, 0, 7] = INF
    c.v[:, 1, 0, 7] = -INF
    out = c.run()[..., c.heads(0), 7]
    both = [i for i in range(N) if masks[i] & 2]
    one = [i for i in range(N) if not masks[i] & 2]
    assert bool(torch.isnan(out[0, both]).all()) and bool((out[0, one] == INF).all())
    assert bool((out[1, both] == -INF).all()) and bool(torch.isfinite(out[1, one]).all())
