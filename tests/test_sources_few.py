"""Rules of the sources of the calls for few tokens that no run shows reliably: how memory is handed over (CPU only)."""
import re

from test_sources import body, source


def test_no_block_of_a_cluster_writes_to_another_before_that_one_has_started():
    """Every block arrives at the cluster's barrier where it starts and waits there ahead of its first remote store."""
    kernel = body(source("pw_few.cu"), "page_linear_kernel(const __grid_constant__")
    arrive, wait, store = (kernel.index(s) for s in ("cluster_arrive()", "cluster_wait()", "store_to_rank("))
    assert arrive < wait < store
    # the wait stands under nothing but "there is a cluster, and this block has not waited yet"
    guard = re.search(r"if \(([^()]*)\) \{\s*cluster_wait\(\);", kernel)
    assert guard and guard.group(1) == "a.split > 1 && !met"
    assert kernel.index("stage_operand") < wait < kernel.index("u0 = first")
