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


# ---- products of many tokens -----------------------------------------------------------------------

def centred_product(x, block, bits):
    """(x . w^T, bound) where code - 2^(bits - 1), times the scale in two fp16 numbers, is multiplied, and the rest of the
    weight with the sum of a group's operand.

    Twice K / 16 accumulations of at most two half steps, K / 128 groups, and the joins of plain_few.product."""
    c, s, z = (m[:, :x.shape[1]] for m in block)
    middle = 2.0 ** (bits - 1) if bits < 16 else 0.0
    size = np.abs(x) @ (np.abs((c - middle) * s) + np.abs(z) + middle * np.abs(s)).T
    return x @ (c * s + z).T, size * (x.shape[1] / 4 + x.shape[1] / 128 + 64) * 2.0 ** -24


def many_tokens(ctx, x, pages, sizes, dtype):
    launches = ctx.pw_launch_count()
    out = ctx.pw_page_linear(x, pages, out_features=sizes, out_dtype=dtype)
    assert ctx.pw_launch_count() - launches == 3 and ctx.pw_last_device_status() == 0
    return out


@pytest.mark.parametrize("T,K,sizes,formats", [(64, 4096, [6000], ["2"]), (33, 8192, [2500, 2000], ["4", "4"]), (130, 2050, [3129, 64], ["3", "4"]),
                                               (70, 14336, [1128], ["8"]), (600, 1000, [1260], ["p4"]), (12000, 640, [100], ["p2"]),
                                               (2000, 900, [700, 33], ["p3", "16"]), (64, 4096, [6000], ["4"]),
                                               (64, 4096, [6000], ["p4"]), (48, 4200, [9700], ["4"]), (48, 4200, [9700], ["p4"]),
                                               (20, 8192, [6000], ["8"]), (17, 4200, [9700], ["16"]), (48, 14336, [2300], ["p3"])])
@pytest.mark.parametrize("dtype,share", [(F16, 0.02), (BF16, 0.005)])
def test_many_tokens_round_nothing_but_the_output(ctx, T, K, sizes, formats, dtype, share):
    """Weights are not rounded to fp16: see test_few_outputs_are_a_neighbour_of_the_rounded_definition for the share."""
    g = gen(T + K)
    pages = [plain.make_page(ctx, block_weights(g, n, K), f) for n, f in zip(sizes, formats)]
    x = operand(g, T, K, pitch=up(K))
    out = many_tokens(ctx, x, pages, sizes, dtype)
    parts = [centred_product(f64(x), [m[:n] for m in plain.stored(ctx, p)], p.bits) for n, p in zip(sizes, pages)]
    want, bound = (np.concatenate([p[i] for p in parts], 1) for i in (0, 1))
    check(out, want, bound, dtype)
    moved = torch.from_numpy(want).to(dtype).cuda() != out
    assert float(moved.double().mean()) <= share


@pytest.mark.parametrize("fmt", ["8", "4", "3", "2", "p4", "p3", "p2"])
def test_extreme_groups_of_many_tokens(ctx, fmt):
    """Groups that span nearly all of fp16's range, its subnormals, one value, zeros; operands at both ends; tokens that are not
    finite."""
    T, K, N = 2000, 600, 1500
    g = gen(17)
    w = normal(g, up(N), up(K))
    w[:, :128] *= 65000.0 / w[:, :128].abs().amax(1, keepdim=True)
    w[:, 100] = 65504.0
    w[:, 101] = -65504.0
    w[:, 128:256] *= 2.0 ** -18
    w[:, 256:384] = 0.75
    w[:, 384:512] = 0
    page = plain.make_page(ctx, w.half(), fmt)
    x = operand(g, T, K, pitch=up(K))
    x[0] *= 2.0 ** -20
    x[1] *= 60000.0 / x[1].abs().max()
    x[2] = 0
    x[3:40, :128] = 0                              # the other groups show
    out = many_tokens(ctx, x, [page], [N], BF16)
    check(out, *centred_product(f64(x), [m[:N] for m in plain.stored(ctx, page)], page.bits), BF16)
    assert torch.all(out[2] == 0)
    y = x.clone()
    y[50, 77], y[60, 300] = float("nan"), float("-inf")
    odd = many_tokens(ctx, y, [page], [N], BF16)
    rest = [t for t in range(T) if t not in (50, 60)]
    assert torch.equal(odd[rest], out[rest]) and not torch.isfinite(odd[[50, 60]]).any()


# ---- a wait that runs out --------------------------------------------------------------------------

@pytest.mark.parametrize("F", [768, 3584])
def test_a_meeting_that_runs_out_is_reported_and_leaves_nothing_behind(F):
    """The last CTA comes to the meeting of all CTAs when its own wait there, of some milliseconds, has run out; with the down
    blocks' columns in parts (short blocks) and in one piece.  Calls queued behind are whole, read or unread status."""
    layer = Layer(20, 2, 256, F, MIX, seed=8, k=4)
    c = layer.ctx
    x, l = layer.tokens(5), layer.logits(5)
    good = c.pw_moe_forward_few(0, x, l, 4)
    layer.check(good, x, plain.routing(f64(l), 4))
    for _ in range(2):
        c.pw_debug_set_wait(polls=200, hook=1)
        c.pw_moe_forward_few(0, x, l, 4)
        torch.cuda.synchronize()
        assert c.pw_last_device_status() == 8 and c.pw_last_device_status() == 0
        c.pw_moe_forward_few(0, x, l, 4)
        c.pw_moe_forward_few(0, x, l, 4)
        c.pw_debug_set_wait(polls=0, hook=0)
        behind = [c.pw_moe_forward_few(0, x, l, 4) for _ in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(y, good) for y in behind)
        assert c.pw_last_device_status() == 8 and c.pw_last_device_status() == 0
        assert torch.equal(c.pw_moe_forward_few(0, x, l, 4), good)
    assert c.pw_last_device_status() == 0
    c.close()


# ---- pages that no block of fp16 weights makes -----------------------------------------------------

@pytest.mark.parametrize("bits", [8, 4, 3, 2])
def test_scales_of_any_sign_and_size(ctx, bits):
    """Imported pages: scales that are zero, negative, subnormal, and as large as the many-token way takes them."""
    rows, cols, T = 1280, 1024, 1000
    g = gen(bits)
    raw = B.Page(rows, cols, bits, ctx.device, B.PW_LAYOUT_CANONICAL)
    raw.codes.copy_(torch.randint(0, 256, raw.codes.shape, generator=g, device="cuda", dtype=torch.int32).to(torch.uint8))
    s = normal(g, rows, cols // 128)
    s[:, 0] = 0
    s[:, 1] *= 2.0 ** -20
    s[:, 2] = 131008.0 / 2 ** bits * torch.sign(s[:, 2])
    s[:, 3] = 2.0 ** -24 * torch.round(8 * s[:, 3])
    raw.scales.copy_(s.half().reshape(raw.scales.shape))
    raw.zps.copy_((normal(g, rows, cols // 128) * 3).half().reshape(raw.zps.shape))
    page = ctx.pw_import_page(raw)
    x = operand(g, T, cols)
    x[:500, 256:384] = 0                           # without the largest group, so that the others show
    block = plain.stored(ctx, page)
    check(many_tokens(ctx, x, [page], [rows], BF16), *centred_product(f64(x), block, bits), BF16)
    check(ctx.pw_page_linear(x[:7], [page], out_dtype=F32), *plain.product(f64(x[:7]), block), F32)
    check(ctx.pw_page_linear(x[600:607], [page], out_dtype=F32), *plain.product(f64(x[600:607]), block), F32)


@pytest.mark.parametrize("T,dtype", [(3, F32), (13, BF16)])
def test_an_h_beyond_fp16_makes_its_token_infinite_and_no_other(mixed, T, dtype):
    """As in the call for batches, whose operand is fp16 too; the largest that fits gives what it should."""
    x, l = mixed.tokens(T), mixed.logits(T)
    want = mixed.ctx.pw_moe_forward_few(0, x, l, 3, out_dtype=dtype)
    pairs = all_pairs(mixed, l, 3)
    g, u = (plain.product(f64(x[1:2]), mixed.blocks[mixed.E][k])[0] for k in (0, 1))   # of a shared expert: every token has it
    y = x.clone()
    for scale, fits in ((64.0, True), (20000.0, False)):
        y[1] = (x[1].float() * scale).half()
        h = np.abs(np.concatenate([(a * scale) / (1 + np.exp(np.clip(-a * scale, -700, 700))) * b * scale for a, b in zip(g, u)]))
        assert (h.max() < 60000) == fits
        out = mixed.ctx.pw_moe_forward_few(0, y, l, 3, out_dtype=dtype)
        rest = [t for t in range(T) if t != 1]
        assert torch.equal(out[rest], want[rest])
        if not fits:
            assert not torch.isfinite(out[1]).any() and not torch.isfinite(mixed.ctx.pw_moe_forward(0, y, l, 3)[1]).any()
    assert pairs and mixed.ctx.pw_last_device_status() == 0
