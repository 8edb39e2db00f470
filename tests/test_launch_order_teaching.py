"""Order of dependent kernels of the calls that teach a probe (no GPU), as test_launch_order.py checks it
for the others: where a kernel waits for the work in front, lets the next one start, and what it reads before."""
import re

import pytest

from test_launch_order import KERNELS

# The first kernels of their calls: sp_norm, sp_norm_backward, sp_vocab_loss with more than 256 tokens or on CUDA cores and
# sp_vocab_loss_backward, sp_attend_tree_backward on CUDA cores and with more than 16 nodes on tensor cores.
FIRST = ["norm_kernel", "norm_loop_kernel", "norm_back_kernel", "norm_back_loop_kernel", "vocab_keep_kernel",
         "tree_back_rows_kernel", "tree_back_rows_tc_kernel"]
# Behind them, and waiting before they read anything.
BEHIND = ["norm_gain_kernel", "vocab_finish_loss_kernel", "vocab_finish_dh_kernel", "vocab_simt_kernel", "vocab_simt_back_kernel",
          "tree_back_simt_kernel", "tree_back_sum_kernel", "tree_back_tc_sum_kernel"]


@pytest.mark.parametrize("name", FIRST)
def test_a_first_kernel_triggers_after_its_wait(name):
    # kernels behind it read the caller's rows, head, lengths and cache in front of their own waits
    body = KERNELS[name]
    assert body.index("pdl_wait()") < body.index("pdl_trigger()")


@pytest.mark.parametrize("name", FIRST + BEHIND)
def test_nothing_is_read_in_front_of_the_wait(name):
    before = KERNELS[name]
    before = before[:before.index("pdl_wait()")]
    assert not re.search(r"\b(a|args|x)\.\w+\s*\[|\*\s*\(?a\.|load\w*\(|resolve_seq|tree_nodes|\bpart\[|__ldcg", before)


def test_tensor_core_losses_wait_in_every_role_and_ask_for_the_head_alone():
    # the first kernel of a loss of up to 256 tokens, or one behind vocab_keep_kernel, which has waited when it triggers:
    # what is copied in front of the wait is the head's, by the kernel that forms the gradient's logits
    body = KERNELS["vocab_tc_kernel"]
    roles = [body.index(s) for s in ("const uint64_t pol_a", "else if (warp == MMA && rank == 0)", "else if (warp < EPI_WARPS)")]
    for at, end in zip(roles, roles[1:] + [len(body)]):
        role = body[at:end]
        before = role[:role.index("pdl_wait()")]
        assert not re.search(r"a\.rows|a\.targets|a\.grad|count_of|tiles_of|map_a", before)
        copies = re.findall(r"tma_load\w*\([^;]*;", before)
        assert len(copies) == (1 if at == roles[0] else 0) and all("&map_b" in c for c in copies)
    ahead = body[roles[0]:roles[1]]
    assert re.search(r"if \(KIND == GRAD && a\.pad == TM && cl < ceil_div\(piece, tn\)\) \{\s*pre =", ahead)
    assert body.index("pdl_trigger()") > body.rindex("__syncthreads()") > body.rindex("pdl_wait()")


def test_blocks_of_the_attention_without_a_share_leave_others_that_wait():
    # the kernel that forms the nodes' products waits at once; behind a kernel that has waited before it triggered,
    # surplus blocks leave without: block group 0 has a share whatever the lengths, and its softmax and
    # row warps wait before they read that kernel's results
    body = KERNELS["tree_back_tc_kernel"]
    first = body.index("if (NODES) pdl_wait();")
    assert first < body.index("back_prefix(") < body.index("if (grp >= n_grp) return;")
    assert not re.search(r"\breturn\b", body[:first])
    rest = body[body.index("if (grp >= n_grp) return;"):]
    softmax, rows = rest.index("if (warp < 8)"), rest.index("else if (warp < MMA)")
    for role, read in ((rest[softmax:rows], "args.stat"), (rest[rows:rest.index("copy_codes")], "args.stat")):
        assert role.index("if (!NODES) pdl_wait();") < role.index(read)
    assert body.index("pdl_trigger()") > body.rindex("__syncthreads()")
