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


# ---- what the layer keeps of h ---------------------------------------------------------------------

def layer_of_two(x, blocks, pairs):
    """(out, bound) of the layer as in plain_few.layer, for an h in two fp16 numbers, the second times 2^11.

    The first is off by at most half a step, 2^-11 of h, and below 2^-14 by 2^-25; the second holds what it leaves to half a
    step of that, 2^-22 of h, or to half of its own smallest step over 2^11, 2^-36.  silu's fast exponential overflows below
    -88 only, which the tests that use this do not meet."""
    out, bound = np.zeros_like(x), np.zeros_like(x)
    for t, e, gate in pairs:
        g, dg = plain.product(x[t:t + 1], blocks[e][0])
        u, du = plain.product(x[t:t + 1], blocks[e][1])
        assert g.min() > -80
        silu = g / (1.0 + np.exp(-g))
        h = silu * u
        # the slope of silu is at most 1.1; its fast exponential and division: a few units of 2^-21
        dh = (1.1 * dg + np.abs(silu) * 2.0 ** -19) * (np.abs(u) + du) + np.abs(silu) * du
        dh = dh + np.maximum((np.abs(h) + dh) * HALF_STEP[F16] ** 2, 2.0 ** -36)
        y, dy = plain.product(h, blocks[e][2])
        c, s, z = blocks[e][2]
        out[t] += gate * y[0]
        bound[t] += abs(gate) * (dy[0] + (dh @ np.abs(c * s + z).T)[0] * 1.001 + np.abs(y[0]) * 2.0 ** -20)
    return out, bound


@pytest.fixture(scope="module")
def mixed():
    layer = Layer(8, 2, 256, 384, MIX, seed=31)
    yield layer
    layer.ctx.close()


def all_pairs(layer, logits, k):
    T = logits.shape[0]
    return plain.routing(f64(logits), k) + [(t, layer.E + s, 1.0) for t in range(T) for s in range(layer.ns)]


@pytest.mark.parametrize("T", [1, 4, 5, 8, 9, 12, 16])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_the_output_is_rounded_once(mixed, T, dtype):
    """Whatever the output's type and the number of tokens, nothing before its rounding shows."""
    x, l = mixed.tokens(T), mixed.logits(T)
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3, out_dtype=dtype)
    check(out, *layer_of_two(f64(x), mixed.blocks, all_pairs(mixed, l, 3)), dtype)


@pytest.mark.parametrize("T", [3, 16])
@pytest.mark.parametrize("scale", [0.1, 0.01, 1e-3])
def test_a_small_h_keeps_its_bits(mixed, T, scale):
    """h is about scale^2 / 4: at 1e-3 its first number has no more than two bits."""
    x, l = (mixed.tokens(T).float() * scale).half(), mixed.logits(T)
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3)
    check(out, *layer_of_two(f64(x), mixed.blocks, all_pairs(mixed, l, 3)), F32)


@pytest.mark.parametrize("T", [4, 12, 16])
@pytest.mark.parametrize("dtype,share", [(F16, 0.02), (BF16, 0.005)])
def test_few_outputs_are_a_neighbour_of_the_rounded_definition(mixed, T, dtype, share):
    """An error d of a value moves its rounding with probability d / step.  Sums in fp32 (some hundred additions, each off by
    2^-25 of the whole or so, at random) and an h of 22 bits make d about 1e-6 of the outputs' size; a step is 2^-8 to 2^-7 of
    a bf16 value, 2^-11 to 2^-10 of an fp16 one, less for the values near zero: about one in a thousand, and four in a
    thousand, move.  With d = 2e-4, an h of 11 bits, 3 % and 28 % would."""
    x, l = mixed.tokens(T), mixed.logits(T)
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3, out_dtype=dtype)
    want, _ = layer_of_two(f64(x), mixed.blocks, all_pairs(mixed, l, 3))
    moved = torch.from_numpy(want).to(dtype).cuda() != out
    assert float(moved.double().mean()) <= share
