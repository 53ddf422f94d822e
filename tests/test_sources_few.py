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


def test_a_product_reads_nothing_before_it_waits_for_the_kernel_ahead():
    """The kernel directly ahead, of whichever context or stream, may be the one that writes the page.  Ahead of the wait
    there are only requests to the L2 cache, which hand no data over."""
    kernel = body(source("pw_few.cu"), "page_linear_kernel(const __grid_constant__")
    wait = kernel.index("grid_dep_sync();")
    assert len(re.findall(r"grid_dep_sync\(\)", kernel)) == 1 and kernel[:wait].count("for (") == 0
    lambdas = "".join(re.findall(r"auto \w+ = \[&\]\(\).*?\n  \};", kernel[:wait], re.S))
    ahead = kernel[:wait]
    for part in re.findall(r"auto \w+ = \[&\]\(\).*?\n  \};", ahead, re.S):
        ahead = ahead.replace(part, "")
    assert "auto ask_next" in lambdas and "auto more" in lambdas
    assert re.findall(r"\b(\w+)(?:<\w+>)?\(f, lane\)", ahead) == ["prefetch_steps"]
    for call in ("ask_next(", "ask<", "ask_any", "cp16", "stage_operand", "load1"):
        assert call not in ahead, call
    request = body(source("pw_stream.cuh"), "void prefetch_steps(")
    assert re.findall(r"asm volatile\(\"(\S+)", request) == ["prefetch.global.L2"] and "cp16" not in request


def test_no_note_of_written_pages_decides_how_a_product_is_launched():
    """Such a note could be lost: to another stream, to a capture, to another context."""
    for name in ("pw_few.cu", "pw_quant.cu", "pw_planes.cu", "pw_common.cuh"):
        assert "page_write" not in source(name)


def test_notes_of_the_layer_are_read_by_all_lanes_before_any_lane_writes_there():
    """The sums of the second phase lie where the notes are, and a lane clears what others have noted."""
    kernel = body(source("pw_few_layer.cu"), "few_layer_kernel(const __grid_constant__")
    read, clear = kernel.index("lds8(notes"), kernel.index("own[i] = 0.f")
    between = kernel[read:clear]
    # outside of every loop and branch: at the depth of braces of the reading
    depth, found = 0, False
    for part in re.findall(r"[{}]|__syncwarp\(\);", between):
        depth += {"{": 1, "}": -1}.get(part, 0)
        found |= part == "__syncwarp();" and depth == 0
    assert found
