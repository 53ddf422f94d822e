"""Rules of the kernels' sources that no run shows reliably: how memory is handed over (CPU only)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_16184_b200", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def body(text, start):
    """From `start` to the end of the braces that follow it."""
    at = text.index(start)
    i = text.index("{", at)
    depth, j = 1, i + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        j += 1
    return text[at:j]


def test_a_wait_that_a_vote_decides_orders_memory():
    """A lane whose own look at a barrier failed acquires nothing by a vote; __syncwarp hands it what the others saw."""
    text = source("pw_linear.cu")
    vote = body(text, "bool warp_saw(")
    assert vote.index("__any_sync") < vote.index("__syncwarp")
    wait = body(text, "bool mbar_wait(")
    returns = re.findall(r"if \(([^;]*)\) return true;", wait)
    assert len(returns) == 2 and all(r.startswith("warp_saw(") for r in returns)


def test_sums_of_other_blocks_are_acquired_at_cluster_scope():
    text = source("pw_linear.cu")
    waits = re.findall(r"mbar_wait(<\w+>)?\(smem_u32\(&sums_in\)", text)
    assert waits == ["<true>"]
    assert "try_wait.parity.acquire.cluster" in body(text, "bool mbar_look(")


def test_first_kernels_of_the_layer_read_the_callers_buffers_through_plain_pointers():
    """Logits, ids and gates may come from the kernel directly ahead, which may still run when a dependent one is placed:
    `const __restrict__` would let the compiler read them through the non-coherent path."""
    text = source("pw_route.cu")
    for name in ("logits", "ids_in", "gates_in"):
        declared = re.findall(r"const (?:float|int32_t)\*\s*(__restrict__)?\s*%s\b" % name, text)
        assert declared and not any(declared), name


def test_header_says_which_calls_use_the_workspace():
    """Calls of the section around the layer may run at the same time; those that work in the context's workspace stand
    with pw_moe_forward, which says that they may not."""
    header = open(os.path.join(CSRC, "..", "..", "include", "pw.h")).read()
    sections = re.split(r"/\* -{3,} ([^-]+?) -{3,} \*/", header)
    where = {name: text for name, text in zip(sections[1::2], sections[2::2])}
    calls = {name: set(re.findall(r"^pw_status (pw_[a-z_]+)\(", text, re.M)) for name, text in where.items()}
    assert calls["around the layer"] == {"pw_quantize_scaled", "pw_add_rmsnorm", "pw_scaled_linear", "pw_route_tokens"}
    assert {"pw_moe_forward", "pw_moe_forward_routed", "pw_moe_forward_host"} <= calls["forward"]
    assert "two at a time need two contexts" in where["forward"]
