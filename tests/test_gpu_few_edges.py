"""Products on weight pages and the layer for few tokens: calls around one another, and values at the ends of the ranges."""
import numpy as np
import pytest
import torch

from paper_2607_16184_b200 import binding as B

import plain_few as plain
from plain_operators import HALF_STEP, f64
from test_gpu_few import BF16, F16, F32, MIX, Layer, block_weights, check, gen, normal, operand, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    yield c
    c.close()


# ---- pages that change ahead of a product ----------------------------------------------------------

def versions(ctx, n, rows, cols):
    """Blocks of weights, a page that takes them in turn, and what a product of each gives."""
    g = gen(rows)
    blocks, x, page = [block_weights(g, rows, cols) for _ in range(n)], operand(g, 2, cols), B.Page(rows, cols, 4, ctx.device)
    want = []
    for w in blocks:
        ctx.pw_quantize_block(w, 4, dst=page)
        torch.cuda.synchronize()
        want.append(ctx.pw_page_linear(x, [page]))
        torch.cuda.synchronize()
    return blocks, x, page, want


def test_a_page_that_another_context_writes_directly_ahead(ctx):
    blocks, x, page, want = versions(ctx, 6, 512, 2048)
    other = B.Context(1, 8, 0, 256, 512, 16, 2)

    def step(w):
        other.pw_quantize_block(w, 4, dst=page)
        return ctx.pw_page_linear(x, [page])

    for w, y in zip(blocks, want):
        assert torch.equal(step(w), y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [step(w) for w in blocks]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    other.close()


def test_pages_written_on_one_of_many_streams(ctx):
    """Products on many other streams between the write of a page and the product that reads it."""
    blocks, x, page, want = versions(ctx, 5, 640, 1024)
    still = plain.make_page(ctx, block_weights(gen(1), 128, 1024), "8")
    streams = [torch.cuda.Stream() for _ in range(32)]
    home = torch.cuda.Stream()
    torch.cuda.synchronize()
    for w, y in zip(blocks, want):
        ctx.pw_quantize_block(w, 4, dst=page, stream=home)
        for s in streams:
            ctx.pw_page_linear(x, [still], stream=s)
        out = ctx.pw_page_linear(x, [page], stream=home)
        home.synchronize()
        assert torch.equal(out, y)
    torch.cuda.synchronize()


def test_a_page_written_on_another_stream_of_a_graph(ctx):
    """The product's only predecessor in the graph is a kernel of another stream, or one of each."""
    blocks, x, page, want = versions(ctx, 4, 512, 2048)
    side = torch.cuda.Stream()
    for alone in (True, False):
        graph, got, y = torch.cuda.CUDAGraph(), [], torch.zeros(64, device="cuda")
        with torch.cuda.graph(graph):
            for w in blocks:
                side.wait_stream(torch.cuda.current_stream())
                ctx.pw_quantize_block(w, 4, dst=page, stream=side)
                if not alone:
                    y.add_(1.0)
                torch.cuda.current_stream().wait_stream(side)
                got.append(ctx.pw_page_linear(x, [page]))
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_product_captured_between_a_write_and_a_product(ctx):
    blocks, x, page, want = versions(ctx, 4, 512, 2048)
    s = torch.cuda.Stream()
    kept = []
    torch.cuda.synchronize()
    for w, y in zip(blocks, want):
        with torch.cuda.stream(s):
            ctx.pw_quantize_block(w, 4, dst=page)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                inside = ctx.pw_page_linear(x, [page])
            out = ctx.pw_page_linear(x, [page])
            graph.replay()
        s.synchronize()
        assert torch.equal(out, y) and torch.equal(inside, y)
        kept.append(graph)
