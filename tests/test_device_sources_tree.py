"""Rules of the kernel for drafted rows that a run on a GPU does not show, checked on its source: breaking one is a hang or a
write into another CTA's shared memory that takes a rare order of events."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_15750_b200", "csrc")


def _body():
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tc_tree.cuh")).read())
    return src[src.index("k_tree_tc("):]


def test_the_join_is_let_in_behind_the_tmem_allocation():
    body = _body()
    assert body.index("tmem_alloc(") < body.index("__syncthreads();") < body.index("pdl_trigger()")
    assert len(re.findall(r"pdl_trigger\(\)", body)) == 1


def test_every_wait_is_bounded_and_agreed_on():
    """One lane waits alone only in the producer; every other wait is voted on in its warp, and the softmax warps of a group come to
    each of its barriers whatever their waits said."""
    body = _body()
    producer = body[body.index("if (warp == 0) {"):body.index("} else if (warp == 1 || warp == 2) {")]
    rest = body[body.index("} else if (warp == 1 || warp == 2) {"):body.index("if (loads_k > 0 && c.abort_flag != 0)")]
    assert "mbar_wait" not in body                       # (the waits of this kernel are tree_wait and tree_wait_warp)
    assert re.search(r"tree_wait\(", producer) and not re.search(r"tree_wait\(", rest)
    assert len(re.findall(r"tree_wait_warp\(", rest)) >= 6
    softmax = rest[rest.index("else if (warp >= 4)"):]
    # after a wait that ran out a softmax warp leaves the loop only behind a vote of its group
    for m in re.finditer(r"if \(!ok\) break;", softmax):
        before = softmax[:m.start()]
        assert before.rindex("all_agree(") > before.rindex("tree_wait_warp(")
    assert "if (!ok) continue;" in softmax


def test_a_cta_that_gives_up_waits_for_its_copies():
    body = _body()
    drain = body.index("late_flag)")
    flag = body.rindex("c.abort_flag != 0", 0, drain)
    last_role_wait = body.rindex("abort_flag)", 0, flag)
    assert "__syncthreads();" in body[last_role_wait:flag]
    assert "tmem_dealloc(" in body[drain:] and body[drain:].index("__syncthreads();") < body[drain:].index("tmem_dealloc(")


def test_the_ctas_of_a_cluster_leave_together():
    """Two barriers of the cluster, on the one path that all CTAs with keys take: one before the reads from one another's shared
    memory, one behind them."""
    body = _body()
    syncs = [m.start() for m in re.finditer(r"cluster_sync\(\)", body)]
    reads = [m.start() for m in re.finditer(r"tree_remote4?\(", body)]
    assert len(syncs) == 2 and reads and all(syncs[0] < r < syncs[1] for r in reads)
    assert "return;" not in body[body.index("pdl_trigger()"):]
