"""Instructions that want all lanes of a warp together (.aligned: barriers of a cluster or of some warps, TMEM), checked on the source of
the kernel for drafted rows: behind code that some lanes leave out nothing but a statement that waits for the lanes brings them together
again, and a barrier that half a warp comes to is undefined."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_15750_b200", "csrc")


def _body():
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "tc_tree.cuh")).read())
    return src[src.index("k_tree_tc("):]


def _statement_before(body, at):
    return body[:at].rstrip().rsplit("\n", 1)[-1].strip()


def test_lanes_are_together_at_barriers_and_at_the_tmem_allocation():
    body = _body()
    found = 0
    for what in (r"ptx::cluster_sync\(\);", r'asm volatile\("bar\.sync', r"ptx::tmem_alloc\("):
        for m in re.finditer(what, body):
            before = _statement_before(body, m.start())
            assert before.endswith("__syncwarp();") or before.endswith("__syncthreads();"), (what, before)
            found += 1
    assert found == 4


def test_lanes_are_together_at_the_next_read_of_tmem_behind_what_one_lane_does():
    body = _body()
    loop = body[body.index("tree_tmem_ld4(s_col + i, u);"):]
    loop = loop[:loop.index("if (j > 0)")]
    assert re.search(r"if \(lane == 0\) \*reinterpret_cast<float4\*>[^;]*;\s*__syncwarp\(\);\s*\}", loop)


def test_products_that_were_issued_end_before_a_cta_that_gives_up_leaves():
    """A commit behind everything that an issuer has issued, and a wait for it with a limit of its own, between the barrier that all roles
    come to after their last wait and the release of TMEM."""
    body = _body()
    ended = body.index("umma_commit(&c.ended")
    start = body.rindex("if (c.abort_flag != 0", 0, ended)
    wait = body.index("tree_wait_warp(&c.ended", ended)
    assert "warp == 1 || warp == 2" in body[start:ended] and "late_flag" in body[wait:body.index(";", wait)]
    last_role_wait = body.rindex(", abort_flag)", 0, start)
    assert "__syncthreads();" in body[last_role_wait:start]
    assert wait < body.rindex("__syncthreads();", 0, body.index("tmem_dealloc("))
