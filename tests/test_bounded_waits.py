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


def test_vocabulary_epilogue_has_one_verdict():
    # the only barrier between the roles takes the eight warps' verdicts and gives them one, so that all go on
    # or none does, and no warp leaves between its wait and that barrier
    roles = _roles("vocab_tc_kernel", "const uint64_t pol_a")
    assert re.findall(BARRIERS, roles) == ["barrier.cta"] and "barrier.cta.red.and" in roles
    epilogue = roles[roles.index("const auto release_acc"):]
    walks = epilogue[epilogue.index("for (int it = cl"):]
    parts = re.split(r"(ok = wait_acc\(\);|ok = release_acc\(ok\);)", walks)
    assert parts[1::2] == ["ok = wait_acc();", "ok = release_acc(ok);"] * 2
    for between in parts[2::4]:
        assert not re.search(r"\breturn\b|if \(!ok\)|\bok =", between)
    # what a warp leaves by is the common verdict
    assert re.match(r"\s*if \(!ok\) break;", parts[4]) and re.match(r"\s*\}", parts[8])


@pytest.mark.parametrize("role", ["stage_rows<NODES>", "node_products("])
def test_attention_backward_warps_meet_whatever_their_waits_said(role):
    # warps 8 to 11 meet where rows are staged and nodes' products formed: neither stands under a verdict,
    # and the walk over the segments ends by its count alone
    roles = _roles("tree_back_tc_kernel", "} else if (warp < MMA) {")
    roles = roles[:roles.index("} else if (EIGHT && warp >= K_WARP)")]
    assert role in roles and not re.search(r"\bbreak\b", roles)
    assert "bool ok = n_seg == 0 || load(0);" in roles and "ok = load(j + 1) && ok;" in roles
    assert re.search(r"for \(int j = 0; j < n_seg; \+\+j\) \{\s*if \(j \+ 1 < n_seg\) ok = load\(j \+ 1\) && ok;", roles)


def test_stages_asked_for_in_front_are_not_waited_for():
    # rank 1 asks for its part of W in front of the count and, with few tokens, copies nothing else: rank 0
    # may have used the stage, and released it on both CTAs, before rank 1 would look whether it is free
    body = KERNELS["vocab_tc_kernel"]
    loads = body[body.index("pre = min(STAGES"):body.index("mbar_wait_drain(&empty[rg.slot]")]
    waits = re.findall(r"if \(([^;{]*?)mbar_wait\(&empty\[s\]", loads)
    assert waits == ["filled >= pre && !"]


class _Barrier:
    def __init__(self):
        self.phase = 0  # completed phases

    def passes(self, parity):
        return self.phase % 2 != parity


@pytest.mark.parametrize("blocks", [1, 2, 6, 7, 13])
@pytest.mark.parametrize("pre", [0, 1, 6])
@pytest.mark.parametrize("rank1_lags", [False, True])
def test_the_ring_of_a_pair_comes_to_its_end(blocks, pre, rank1_lags):
    """The two copying threads and the MMA warp as steps that run until each waits: rank 1 copies W alone."""
    stages, pre = 6, min(pre, blocks)
    empty = [[_Barrier() for _ in range(stages)] for _ in range(2)]
    got = [[0] * stages for _ in range(2)]  # parts of a stage that have come: rank 0's A and W, rank 1's W
    want = [2, 1]

    def copies(rank):
        for i in range(pre):
            got[rank][i] += 1
        yield
        for i in range(blocks):
            s = i % stages
            while i >= pre and not empty[rank][s].passes((i // stages & 1) ^ 1):
                yield
            got[rank][s] += want[rank] - (1 if i < pre else 0)
            yield
        for j in range(stages):  # the last use of every stage
            use = blocks - 1 - (blocks - 1 - j) % stages if j < blocks else -1
            while use >= 0 and not empty[rank][j].passes(use // stages & 1):
                yield

    def mma():
        for i in range(blocks):
            s = i % stages
            while [got[0][s], got[1][s]] != [(i // stages + 1) * w for w in want]:
                yield
            for rank in range(2):
                empty[rank][s].phase += 1
            yield

    tasks = [copies(0), mma(), copies(1)]
    steps = 0
    while tasks:
        steps += 1
        assert steps < 10000, "a wait that nothing ends"
        for t in list(tasks):
            if rank1_lags and len(tasks) == 3 and t is tasks[2] and steps % 40 not in (1,):
                continue
            if next(t, "end") == "end":
                tasks.remove(t)
