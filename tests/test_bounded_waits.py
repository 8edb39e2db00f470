"""Waits with a limit (no GPU): a warp whose wait ran out goes its own way, so that between the
roles' beginning and the block's end no warp may stand at a barrier, which has no limit, where
another warp's own verdict decides whether it comes.  A hang shows only on a failing GPU, so the
source is read."""
import re

import pytest

from test_launch_order import KERNELS


def _roles(name, first):
    """The part of a kernel in which warps do different things: from its first role to the last meeting."""
    body = KERNELS[name]
    return body[body.index(first):body.rindex("__syncthreads()")]


BARRIERS = r"bar\.sync|barrier\.cta|barrier\.sync|named_sync|__syncthreads|cluster_sync"


def test_vocabulary_kernel_waits_have_a_limit():
    roles = _roles("vocab_tc_kernel", "const uint64_t pol_a")
    assert "wait_acc" in roles and "release_acc" in roles
    assert not re.search(BARRIERS, roles)


def test_vocabulary_accumulators_are_released_by_every_warp_that_reads_them():
    # each of the eight warps of both CTAs arrives for itself: the count that the barriers are made with
    body = KERNELS["vocab_tc_kernel"]
    assert re.search(r"mbar_init\(&acc_empty\[i\], 2 \* EPI_WARPS\)", body)
    release = body[body.index("release_acc = "):]
    release = release[:release.index("};")]
    assert re.search(r"tc_fence_before\(\);\s*__syncwarp\(\);\s*if \(lane == 0\) mbar_arrive_remote\(", release)


@pytest.mark.parametrize("role", ["stage_rows<NODES>", "node_products("])
def test_attention_backward_warps_meet_whatever_their_waits_said(role):
    # warps 8 to 11 meet where rows are staged and nodes' products formed: neither stands under a verdict,
    # and the walk over the segments ends by its count alone
    roles = _roles("tree_back_tc_kernel", "} else if (warp < MMA) {")
    roles = roles[:roles.index("} else if (EIGHT && warp >= K_WARP)")]
    assert role in roles and not re.search(r"\bbreak\b", roles)
    assert "bool ok = n_seg == 0 || load(0);" in roles and "ok = load(j + 1) && ok;" in roles
    assert re.search(r"for \(int j = 0; j < n_seg; \+\+j\) \{\s*if \(j \+ 1 < n_seg\) ok = load\(j \+ 1\) && ok;", roles)
