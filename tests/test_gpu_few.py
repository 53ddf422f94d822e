"""Products on weight pages and the layer for few tokens against their definitions in 64 bits."""
import threading

import numpy as np
import pytest
import torch

from paper_2607_16184_b200 import binding as B

import plain_few as plain
from plain_operators import f64

pytestmark = pytest.mark.gpu
F16, F32, BF16 = torch.float16, torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    yield c
    c.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def up(n):
    return -(-n // 128) * 128


def block_weights(g, n, k, fill=0.0):
    """fp16 weights of a page with room for [n, k]; `fill` behind them."""
    w = torch.full((up(n), up(k)), fill, device="cuda")
    w[:n, :k] = normal(g, n, k) * 0.02
    return w.half()


def operand(g, T, K, pitch=None):
    x = torch.zeros(T, pitch or -(-K // 8) * 8, dtype=F16, device="cuda")[:, :K]
    x.copy_(normal(g, T, K))
    return x


def check(got, want, bound, dtype):
    d = np.abs(f64(got) - want)
    limit = plain.rounded(want, bound, dtype)
    assert np.all(d <= limit), "%g of the bound" % np.max(d / limit)


# ---- products --------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,K,N", [(1, 128, 32), (1, 1, 1), (2, 300, 33), (8, 640, 129), (9, 2050, 60), (17, 257, 40)])
@pytest.mark.parametrize("fmt", plain.FORMATS)
def test_product(ctx, fmt, T, K, N):
    g = gen(T + K)
    page = plain.make_page(ctx, block_weights(g, N, K), fmt)
    x = operand(g, T, K)
    out = ctx.pw_page_linear(x, [page], out_features=[N], out_dtype=F32)
    check(out, *plain.product(f64(x), [m[:N] for m in plain.stored(ctx, page)]), F32)


@pytest.mark.parametrize("T,K,N,fmt", [(8, 14336, 70, "3"), (5, 20000, 33, "16"), (8, 33000, 40, "8"), (1, 60001, 40, "4"), (12, 9000, 300, "p4"),
                                       (70, 500, 500, "4"), (1300, 16, 8, "8"), (3, 4096, 9000, "2")])
def test_product_of_long_rows_and_many_tokens(ctx, T, K, N, fmt):
    """Columns split over a cluster, passes of fewer tokens, more passes than clusters, more units than teams."""
    g = gen(K)
    page = plain.make_page(ctx, block_weights(g, N, K), fmt)
    x = operand(g, T, K)
    out = ctx.pw_page_linear(x, [page], out_features=[N], out_dtype=F32)
    check(out, *plain.product(f64(x), [m[:N] for m in plain.stored(ctx, page)]), F32)


@pytest.mark.parametrize("dtype,bias_type", [(F16, F32), (BF16, BF16), (F32, F16), (F16, None)])
@pytest.mark.parametrize("T", [1, 6, 11])
def test_several_pages_bias_and_strides(ctx, dtype, bias_type, T):
    """Pages of different formats side by side; what lies between the rows stays."""
    g = gen(T)
    sizes, formats, K = [200, 64, 1, 130], ["4", "8", "16", "p3"], 389
    pages = [plain.make_page(ctx, block_weights(g, n, K), f) for n, f in zip(sizes, formats)]
    x = operand(g, T, K, pitch=520)
    bias = None if bias_type is None else normal(g, sum(sizes)).to(bias_type)
    whole = torch.full((T, sum(sizes) + 13), 7.0, dtype=dtype, device="cuda")
    out = ctx.pw_page_linear(x, pages, out_features=sizes, bias=bias, out=whole[:, :sum(sizes)])
    parts = [plain.product(f64(x), [m[:n] for m in plain.stored(ctx, p)]) for n, p in zip(sizes, pages)]
    want, bound = (np.concatenate([p[i] for p in parts], 1) for i in (0, 1))
    if bias is not None:
        want = want + f64(bias)
        bound = bound + (np.abs(want) + bound) * 2.0 ** -24
    check(out, want, bound, dtype)
    assert torch.all(whole[:, sum(sizes):] == 7.0)


def test_what_a_page_holds_past_the_block_does_not_count(ctx):
    g = gen(3)
    w = block_weights(g, 50, 300, fill=9.0)
    w[:50, :300] = block_weights(g, 50, 300)[:50, :300]
    x = operand(g, 3, 300)
    for fmt in ("16", "8", "p2"):
        page = plain.make_page(ctx, w, fmt)
        whole = torch.full((3, 64), 5.0, device="cuda")
        out = ctx.pw_page_linear(x, [page], out_features=[50], out=whole[:, :50])
        check(out, *plain.product(f64(x), [m[:50] for m in plain.stored(ctx, page)]), F32)
        assert torch.all(whole[:, 50:] == 5.0)


@pytest.mark.parametrize("fmt", plain.FORMATS)
def test_extreme_values(ctx, fmt):
    """Constant groups, groups at both ends of fp16's range, operands at both ends; a token with NaN or infinity keeps it to
    itself."""
    g = gen(4)
    w = block_weights(g, 128, 512).float()
    w[:, :128] = 0.75
    w[:, 128:256] *= 2.0 ** -16
    w[:, 256:384] *= 40000.0 / w[:, 256:384].abs().max()
    w[3] = 0
    page = plain.make_page(ctx, w.half(), fmt)
    x = operand(g, 6, 512)
    x[0] *= 2.0 ** -20                             # subnormal operands
    x[1] *= 60000.0 / x[1].abs().max()
    x[2] = 0
    out = ctx.pw_page_linear(x, [page], out_dtype=F32)
    check(out, *plain.product(f64(x), plain.stored(ctx, page)), F32)
    assert torch.all(out[2] == 0)
    y = x.clone()
    y[4, 77], y[5, 300] = float("nan"), float("inf")
    odd = ctx.pw_page_linear(y, [page], out_dtype=F32)
    assert torch.equal(odd[:4], out[:4])
    assert torch.isnan(odd[4]).all() and not torch.isfinite(odd[5, w[:, 300] != 0]).any()


def test_products_repeat(ctx):
    """The same bits in every call; a token's row does not depend on where it stands."""
    g = gen(5)
    pages = [plain.make_page(ctx, block_weights(g, 700, 900), f) for f in ("4", "8")]
    x = operand(g, 8, 900)
    out = ctx.pw_page_linear(x, pages, out_dtype=F32)
    for _ in range(3):
        assert torch.equal(ctx.pw_page_linear(x, pages, out_dtype=F32), out)
    y = operand(g, 8, 900)
    y[:, :] = x.flip(0)
    assert torch.equal(ctx.pw_page_linear(y, pages, out_dtype=F32).flip(0), out)


@pytest.mark.parametrize("T,K,sizes,formats,kernels", [
    (1200, 128, [40], ["4"], 1), (700, 300, [130, 1, 300], ["16", "p3", "8"], 1), (64, 4096, [6000], ["2"], 3), (300, 1000, [1260], ["p4"], 1),
    (600, 1000, [1260], ["p4"], 3), (130, 2050, [3129, 64], ["3", "4"], 3), (600, 640, [100], ["p2"], 1), (1000, 40, [133], ["16"], 1),
    (70, 14336, [1128], ["8"], 3), (33, 8192, [2500, 2000], ["4", "4"], 3), (4500, 300, [130, 1, 300], ["16", "p3", "8"], 3),
    (12000, 640, [100], ["p2"], 3), (70000, 40, [133], ["16"], 3)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_product_of_many_tokens(ctx, T, K, sizes, formats, kernels, dtype):
    """16-bit outputs of many tokens: weights are rounded to fp16, half a step each, where that many kernels run."""
    g = gen(T)
    pages = [plain.make_page(ctx, block_weights(g, n, K), f) for n, f in zip(sizes, formats)]
    x, bias = operand(g, T, K, pitch=up(K)), normal(g, sum(sizes)) * 3
    whole = torch.full((T, sum(sizes) + 5), 7.0, dtype=dtype, device="cuda")
    launches = ctx.pw_launch_count()
    out = ctx.pw_page_linear(x, pages, out_features=sizes, bias=bias, out=whole[:, :sum(sizes)])
    assert ctx.pw_launch_count() - launches == kernels and ctx.pw_last_device_status() == 0
    want, bound = [], []
    for n, p in zip(sizes, pages):
        block = [m[:n] for m in plain.stored(ctx, p)]
        y, d = plain.product(f64(x), block)
        w = np.abs(block[0] * block[1] + block[2])[:, :K]
        want.append(y)
        bound.append(d + (0 if p.bits == 16 else np.abs(f64(x)) @ (w * 2.0 ** -11 + 2.0 ** -25).T))
    want, bound = np.concatenate(want, 1) + f64(bias), np.concatenate(bound, 1)
    check(out, want, bound + (np.abs(want) + bound) * 2.0 ** -24, dtype)
    assert torch.all(whole[:, sum(sizes):] == 7.0)
    assert torch.equal(ctx.pw_page_linear(x, pages, out_features=sizes, bias=bias, out_dtype=dtype), out)


def test_many_tokens_in_a_graph_and_on_two_streams(ctx):
    g = gen(31)
    page = plain.make_page(ctx, block_weights(g, 1000, 1024), "4")
    xs = [operand(g, T, 1024) for T in (400, 300)]
    want = [ctx.pw_page_linear(x, [page]) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [[torch.empty_like(w) for _ in range(10)] for w in want]
    for i in range(10):
        for x, s, o in zip(xs, streams, outs):
            ctx.pw_page_linear(x, [page], out=o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, many in zip(want, outs) for o in many)
    out = torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.pw_page_linear(xs[0], [page], out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])


def test_no_tokens(ctx):
    page = plain.make_page(ctx, block_weights(gen(6), 40, 256), "4")
    out = ctx.pw_page_linear(torch.empty(0, 256, dtype=F16, device="cuda"), [page], out_features=[40])
    assert out.shape == (0, 40)


def test_product_in_a_graph_and_on_two_streams(ctx):
    g = gen(7)
    pages = [plain.make_page(ctx, block_weights(g, 3000, 2048), f) for f in ("4", "3")]
    xs = [operand(g, 4, 2048) for _ in range(2)]
    want = [ctx.pw_page_linear(x, [p], out_dtype=F32) for x, p in zip(xs, pages)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(w) for _ in range(8)] for w in want]
    for i in range(8):
        for s, x, p, o in zip(streams, xs, pages, outs):
            ctx.pw_page_linear(x, [p], out=o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, many in zip(want, outs) for o in many)
    x, out = xs[0].clone(), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.pw_page_linear(x, [pages[0]], out=out)
    for src, w in ((xs[1], None), (xs[0], want[0])):
        x.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ctx.pw_page_linear(src, [pages[0]], out_dtype=F32) if w is None else w)


def test_calls_of_two_threads(ctx):
    g = gen(8)
    page = plain.make_page(ctx, block_weights(g, 500, 1024), "4")
    xs = [operand(g, 2, 1024) for _ in range(2)]
    want = [ctx.pw_page_linear(x, [page], out_dtype=F32) for x in xs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        s = torch.cuda.Stream()
        for _ in range(50):
            out = ctx.pw_page_linear(xs[i], [page], out_dtype=F32, stream=s)
            s.synchronize()
            if not torch.equal(out, want[i]):
                wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("T,dtype", [(5, F32), (40, F16)])
def test_a_token_that_is_not_finite_stays_alone(ctx, T, dtype, bad):
    g = gen(5)
    pages = [plain.make_page(ctx, block_weights(g, n, 640), f) for n, f in ((100, "4"), (64, "8"), (33, "16"), (40, "p3"))]
    x = operand(g, T, 600)
    want = ctx.pw_page_linear(x, pages, out_dtype=dtype)
    x[3, 77] = bad
    got = ctx.pw_page_linear(x, pages, out_dtype=dtype)
    assert not torch.any(torch.isfinite(got[3]))
    assert torch.equal(got[[t for t in range(T) if t != 3]], want[[t for t in range(T) if t != 3]])


def test_a_page_that_is_written_directly_ahead(ctx):
    """The product may begin while the kernel ahead of it still runs, but not with a page that kernel writes."""
    g = gen(77)
    blocks = [block_weights(g, 512, 4096) for _ in range(6)]
    x = operand(g, 3, 4096)
    page, demoted = B.Page(512, 4096, 8, ctx.device), B.Page(512, 4096, 4, ctx.device)
    want = []
    for w in blocks:
        ctx.pw_quantize_block(w, 8, dst=page)
        ctx.pw_demote_block(page, 4, dst=demoted)
        torch.cuda.synchronize()
        want.append([ctx.pw_page_linear(x, [p]) for p in (page, demoted)])
        torch.cuda.synchronize()

    def step(w):
        ctx.pw_quantize_block(w, 8, dst=page)
        first = ctx.pw_page_linear(x, [page])
        ctx.pw_demote_block(page, 4, dst=demoted)
        return [first, ctx.pw_page_linear(x, [demoted])]

    for w, two in zip(blocks, want):
        assert all(torch.equal(a, b) for a, b in zip(step(w), two))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [step(w) for w in blocks]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_product_refuses(ctx):
    g = gen(9)
    page = plain.make_page(ctx, block_weights(g, 128, 256), "4")
    x = operand(g, 2, 256)
    for status, call in [(1, lambda: ctx.pw_page_linear(x.float(), [page])), (1, lambda: ctx.pw_page_linear(x, [])),
                         (1, lambda: ctx.pw_page_linear(x.cpu(), [page])), (2, lambda: ctx.pw_page_linear(x.t(), [page])),
                         (2, lambda: ctx.pw_page_linear(x, [page], out_features=[128, 1])), (1, lambda: ctx.pw_page_linear(x, [page], out_features=[0])),
                         (2, lambda: ctx.pw_page_linear(x, [page], out_features=[129])), (2, lambda: ctx.pw_page_linear(x[:, :128], [page])),
                         (2, lambda: ctx.pw_page_linear(x, [page], out=torch.empty(2, 127, device="cuda"))),
                         (1, lambda: ctx.pw_page_linear(x, [page], out=torch.empty(2, 128, dtype=torch.float64, device="cuda"))),
                         (2, lambda: ctx.pw_page_linear(x, [page], bias=torch.empty(127, device="cuda"))),
                         (4, lambda: ctx.pw_page_linear(operand(g, 2, 256, pitch=257), [page])),
                         (5, lambda: ctx.pw_page_linear(x, [ctx.pw_export_page(page)]))]:
        with pytest.raises(B.PwError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(TypeError):
        ctx.pw_page_linear(x, [page], out_features=["a"])
    with pytest.raises(AttributeError):
        ctx.pw_page_linear(x, [x])


# ---- layer -----------------------------------------------------------------------------------------

class Layer:
    """A context with one layer of random weights, and what its pages hold."""

    def __init__(self, E, ns, H, F, formats, seed=0, k=None, max_tokens=16, guard=0):
        g = gen(seed)
        self.ctx = B.Context(1, E, ns, H, F, max_tokens, k or min(E, 8), guard_bytes=guard)
        self.E, self.ns, self.H = E, ns, H
        self.pages, entries = [], []
        for e in range(E + ns):
            three = [plain.make_page(self.ctx, (normal(g, *((H, F) if u == 2 else (F, H))) * 0.05).half(),
                                     "16" if e >= E else formats[(3 * e + u) % len(formats)]) for u in range(3)]
            self.pages.append(three)
            entries += [(0, e, u, p) for u, p in enumerate(three)]
        self.ctx.pw_set_page_table(entries)
        self.blocks = [[plain.stored(self.ctx, p) for p in three] for three in self.pages]
        self.g = g

    def tokens(self, T):
        return normal(self.g, T, self.H).half()

    def logits(self, T):
        return normal(self.g, T, self.E)

    def want(self, x, pairs):
        shared = [(t, self.E + s, 1.0) for t in range(x.shape[0]) for s in range(self.ns)]
        return plain.layer(f64(x), self.blocks, list(pairs) + shared)

    def check(self, out, x, pairs):
        assert self.ctx.pw_last_device_status() == 0
        check(out, *self.want(x, pairs), out.dtype)


MIX = ["16", "4", "8", "3", "2", "p4", "p3", "p2", "4", "4", "8"]


@pytest.fixture(scope="module")
def mixed():
    layer = Layer(8, 2, 256, 384, MIX)
    yield layer
    layer.ctx.close()


@pytest.mark.parametrize("T", [1, 2, 3, 5, 8, 9, 16])
def test_layer(mixed, T):
    x, l = mixed.tokens(T), mixed.logits(T)
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3)
    mixed.check(out, x, plain.routing(f64(l), 3))
    for _ in range(2):
        assert torch.equal(mixed.ctx.pw_moe_forward_few(0, x, l, 3), out)


@pytest.mark.parametrize("fmt", plain.FORMATS)
def test_layer_of_one_format(fmt):
    layer = Layer(4, 0, 384, 256, [fmt], seed=3)
    for T in (1, 7, 16):
        x, l = layer.tokens(T), layer.logits(T)
        layer.check(layer.ctx.pw_moe_forward_few(0, x, l, 2), x, plain.routing(f64(l), 2))
    layer.ctx.close()


@pytest.mark.parametrize("E,ns,H,F,k,T", [(1, 0, 128, 128, 1, 1), (256, 0, 128, 128, 8, 16), (40, 16, 128, 256, 5, 4), (3, 1, 1024, 128, 3, 16),
                                          (5, 0, 128, 2048, 2, 11), (64, 1, 256, 256, 32, 3), (2, 0, 4096, 128, 1, 16)])
def test_layer_shapes(E, ns, H, F, k, T):
    layer = Layer(E, ns, H, F, ["4", "16", "8"], seed=E, k=k)
    x, l = layer.tokens(T), layer.logits(T)
    layer.check(layer.ctx.pw_moe_forward_few(0, x, l, k), x, plain.routing(f64(l), k))
    layer.ctx.close()


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 9, 16])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_layer_keeps_what_its_output_can_show(mixed, T, dtype):
    """The operand of the down blocks is two fp16 numbers where the output is fp32, or fp16 with up to eight tokens."""
    x, l = mixed.tokens(T), mixed.logits(T)
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3, out_dtype=dtype)
    pairs = plain.routing(f64(l), 3) + [(t, mixed.E + s, 1.0) for t in range(T) for s in range(mixed.ns)]
    check(out, *plain.layer(f64(x), mixed.blocks, pairs, parts=2 if dtype == F32 or T <= 8 else 1), dtype)


@pytest.mark.parametrize("T", [1, 2, 4, 7, 8, 9, 13, 16])
def test_layer_whose_down_blocks_are_cut_in_parts(T):
    layer = Layer(20, 4, 256, 768, MIX, seed=6, k=4)
    x = layer.tokens(T)
    for _ in range(3):
        l = layer.logits(T)
        layer.check(layer.ctx.pw_moe_forward_few(0, x, l, 4), x, plain.routing(f64(l), 4))
    layer.ctx.close()


def test_the_room_that_is_promised():
    """T * hidden up to 65536 for 48 pairs, up to 49152 for more."""
    for E, ns, H, k, T in ((8, 0, 4096, 3, 16), (4, 0, 8192, 2, 8), (20, 0, 4096, 8, 12), (18, 0, 16384, 17, 3), (2, 0, 32768, 2, 2)):
        layer = Layer(E, ns, H, 128, ["2"], seed=E, k=k)
        x, l = layer.tokens(T), layer.logits(T)
        layer.check(layer.ctx.pw_moe_forward_few(0, x, l, k), x, plain.routing(f64(l), k))
        layer.ctx.close()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_layer_for_a_given_routing(mixed, dtype):
    """No expert, an expert twice, gates of any size; a row that takes nothing keeps the shared experts'."""
    x = mixed.tokens(6)
    ids = torch.tensor([[0, 1, 2], [-1, -1, -1], [5, 5, 5], [7, -1, 7], [3, 4, 3], [-1, 6, -1]], dtype=torch.int32, device="cuda")
    gates = normal(mixed.g, 6, 3) * 3
    out = mixed.ctx.pw_moe_forward_few_routed(0, x, ids, gates, out_dtype=dtype)
    pairs = [(t, e, float(gates[t, j])) for t, row in enumerate(ids.tolist()) for j, e in enumerate(row) if e >= 0]
    mixed.check(out, x, pairs)


@pytest.mark.parametrize("T", [4, 11])
def test_a_token_of_a_layer_that_is_not_finite_stays_alone(mixed, T):
    x, l = mixed.tokens(T), mixed.logits(T)
    x[2, 5], l[0, :] = float("nan"), float("nan")
    got = mixed.ctx.pw_moe_forward_few(0, x, l, 3)
    assert torch.all(torch.isnan(got[[0, 2]])) and mixed.ctx.pw_last_device_status() == 0
    # (which experts take part is part of the sums' order: the others' bits may change, their values may not)
    rest = [t for t in range(T) if t not in (0, 2)]
    want, bound = mixed.want(x[rest], plain.routing(f64(l[rest]), 3))
    check(got[rest], want, bound, got.dtype)


def test_rows_without_anything_are_zero():
    layer = Layer(4, 0, 128, 128, ["4"], seed=9)
    x = layer.tokens(3)
    ids = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    out = torch.full((3, 128), 5.0, device="cuda")
    layer.ctx.pw_moe_forward_few_routed(0, x, ids, torch.ones(3, 2, device="cuda"), out=out)
    assert torch.all(out == 0) and layer.ctx.pw_last_device_status() == 0
    ids[1, 0] = 2
    layer.ctx.pw_moe_forward_few_routed(0, x, ids, torch.ones(3, 2, device="cuda"), out=out)
    assert torch.all(out[[0, 2]] == 0) and torch.any(out[1] != 0)
    layer.check(out, x, [(1, 2, 1.0)])
    layer.ctx.close()


def test_an_id_that_is_no_expert_is_reported(mixed):
    x = mixed.tokens(2)
    ids = torch.tensor([[1, 8], [-2, 3]], dtype=torch.int32, device="cuda")
    gates = torch.ones(2, 2, device="cuda")
    out = mixed.ctx.pw_moe_forward_few_routed(0, x, ids, gates)
    assert mixed.ctx.pw_last_device_status() == 1
    mixed.check(out, x, [(0, 1, 1.0), (1, 3, 1.0)])


def test_ties_and_masked_logits(mixed):
    x = mixed.tokens(4)
    l = torch.zeros(4, 8, device="cuda")
    l[1, :5] = float("-inf")
    l[2, 6] = float("nan")
    l[3] = torch.finfo(F32).min
    l[3, 5] = 0
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3)
    mixed.check(out, x, plain.routing(f64(l), 3))
    l[2] = float("nan")
    out = mixed.ctx.pw_moe_forward_few(0, x, l, 3)
    assert torch.isnan(out[2]).all() and torch.isfinite(out[[0, 1, 3]]).all()
    mixed.ctx.pw_last_device_status()


def test_layer_agrees_with_the_call_for_batches(mixed):
    """The two differ in one rounding of the weights (half a step of fp16 each) and in the order of sums."""
    x, l = mixed.tokens(16), mixed.logits(16)
    few, batch = mixed.ctx.pw_moe_forward_few(0, x, l, 2), mixed.ctx.pw_moe_forward(0, x, l, 2)
    assert torch.linalg.norm(few - batch) <= 3 * 2.0 ** -11 * torch.linalg.norm(batch)


def test_layer_and_the_calls_for_batches_share_a_workspace(mixed):
    """Neither disturbs the other, and pw_get_routing still tells of the call for batches."""
    x, l = mixed.tokens(16), mixed.logits(16)
    few, batch = mixed.ctx.pw_moe_forward_few(0, x, l, 2), mixed.ctx.pw_moe_forward(0, x, l, 2)
    routing = {k: v.clone() for k, v in mixed.ctx.pw_get_routing(16, 2).items()}
    for _ in range(3):
        assert torch.equal(mixed.ctx.pw_moe_forward_few(0, x[:5].contiguous(), l[:5].contiguous(), 2), mixed.ctx.pw_moe_forward_few(0, x[:5].contiguous(), l[:5].contiguous(), 2))
        assert torch.equal(mixed.ctx.pw_moe_forward_few(0, x, l, 2), few)
        assert all(torch.equal(v, routing[k]) for k, v in mixed.ctx.pw_get_routing(16, 2).items())
        assert torch.equal(mixed.ctx.pw_moe_forward(0, x, l, 2), batch)


def test_a_committed_page_is_read_by_the_next_call():
    layer = Layer(4, 0, 256, 256, ["16"], seed=5)
    x, l = layer.tokens(4), layer.logits(4)
    layer.check(layer.ctx.pw_moe_forward_few(0, x, l, 2), x, plain.routing(f64(l), 2))
    for e, u, bits in ((0, 0, 4), (1, 2, 8), (2, 1, 2), (3, 2, 3)):
        page = layer.ctx.pw_demote_block(layer.pages[e][u], bits)
        layer.ctx.pw_set_page_table([(0, e, u, page)])
        layer.blocks[e][u] = plain.stored(layer.ctx, page)
        layer.check(layer.ctx.pw_moe_forward_few(0, x, l, 2), x, plain.routing(f64(l), 2))
    layer.ctx.close()


@pytest.mark.parametrize("given", [False, True])
def test_observation_taps(given):
    """The same sums as the call for batches notes: masses and counts to a rounding, norms as far as the SwiGLU rows differ."""
    layer = Layer(8, 1, 256, 384, ["4", "8", "16"], seed=6)
    x, l = layer.tokens(12), layer.logits(12)
    ids, gates = layer.ctx.pw_route_tokens(l, 3)
    if given:
        ids[0, 1] = ids[0, 0]                      # a pair that is named twice
        ids[3] = -1
    sums = []
    for few in (True, False):
        acc = layer.ctx.pw_observe(True)
        for _ in range(2):
            if given:
                (layer.ctx.pw_moe_forward_few_routed if few else layer.ctx.pw_moe_forward_routed)(0, x, ids, gates)
            else:
                (layer.ctx.pw_moe_forward_few if few else layer.ctx.pw_moe_forward)(0, x, l, 3)
        sums.append(f64(acc)[0])
        layer.ctx.pw_observe(False)
    a, b = sums
    assert np.array_equal(a[:, 1], b[:, 1])
    assert np.allclose(a[:, [0, 2, 3, 4]], b[:, [0, 2, 3, 4]], rtol=1e-5, atol=1e-6)
    assert np.allclose(a[:, 5:], b[:, 5:], rtol=3 * 2.0 ** -11, atol=1e-6)
    layer.ctx.close()


def test_layer_in_a_graph_and_in_two_contexts_at_once():
    layers = [Layer(8, 1, 512, 512, ["4", "8"], seed=s) for s in (11, 12)]
    x, l = layers[0].tokens(2), layers[0].logits(2)
    want = [y.ctx.pw_moe_forward_few(0, x, l, 2) for y in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    outs = [[torch.empty_like(want[0]) for _ in range(20)] for _ in layers]
    for i in range(20):
        for y, s, o in zip(layers, streams, outs):
            y.ctx.pw_moe_forward_few(0, x, l, 2, out=o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, many in zip(want, outs) for o in many)
    out = torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layers[0].ctx.pw_moe_forward_few(0, x, l, 2, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])
    for y in layers:
        assert y.ctx.pw_last_device_status() == 0
        y.ctx.close()


def test_layer_keeps_to_its_workspace():
    layer = Layer(16, 1, 256, 256, ["4"], seed=13, guard=4096)
    for T in (1, 16):
        x, l = layer.tokens(T), layer.logits(T)
        whole = torch.full((T + 2, 256), 3.0, device="cuda")
        layer.ctx.pw_observe(True)
        layer.ctx.pw_moe_forward_few(0, x, l, 8, out=whole[1:T + 1])
        layer.ctx.pw_observe(False)
        assert torch.all(whole[0] == 3) and torch.all(whole[-1] == 3) and layer.ctx.workspace_guards_intact()
    layer.ctx.close()


def test_layer_refuses(mixed):
    x, l = mixed.tokens(2), mixed.logits(2)
    ids, gates = mixed.ctx.pw_route_tokens(l, 2)
    few, routed = mixed.ctx.pw_moe_forward_few, mixed.ctx.pw_moe_forward_few_routed
    for status, call in [(1, lambda: few(1, x, l, 2)), (1, lambda: few(0, x, l, 0)), (1, lambda: few(0, x, l, 9)), (1, lambda: few(0, x.float(), l, 2)),
                         (2, lambda: few(0, x[:, :128].contiguous(), l, 2)), (2, lambda: few(0, x, l[:1], 2)), (1, lambda: few(0, x, l.half(), 2)),
                         (1, lambda: few(0, x, l, 2, out=torch.empty(2, 256, dtype=torch.int32, device="cuda"))),
                         (2, lambda: few(0, x, l, 2, out=torch.empty(2, 255, device="cuda"))), (1, lambda: routed(0, x, ids.long(), gates)),
                         (2, lambda: routed(0, x, ids, gates[:, :1].contiguous())), (1, lambda: few(0, x.cpu(), l, 2))]:
        with pytest.raises(B.PwError) as e:
            call()
        assert e.value.status == status
    many = Layer(4, 0, 128, 128, ["4"], seed=1, max_tokens=32)
    for T, status in ((17, 1), (33, 1)):
        with pytest.raises(B.PwError) as e:
            many.ctx.pw_moe_forward_few(0, many.tokens(T), many.logits(T), 2)
        assert e.value.status == status
    empty = B.Context(1, 4, 0, 128, 128, 16, 2)
    with pytest.raises(B.PwError) as e:
        empty.pw_moe_forward_few(0, many.tokens(1), many.logits(1), 2)
    assert e.value.status == 5
    wide = Layer(1, 0, 8192, 128, ["2"], seed=2)
    with pytest.raises(B.PwError) as e:
        wide.ctx.pw_moe_forward_few(0, wide.tokens(16), wide.logits(16), 1)
    assert e.value.status == 2
    x, l = wide.tokens(8), wide.logits(8)
    wide.check(wide.ctx.pw_moe_forward_few(0, x, l, 1), x, plain.routing(f64(l), 1))
    for c in (many.ctx, empty, wide.ctx):
        c.close()


# ---- together --------------------------------------------------------------------------------------

@pytest.mark.parametrize("T", [1, 5])
def test_a_decode_step_around_the_layer(T):
    """Norm, projections out of pages, router out of a page, routing, layer, residual and norm, vocabulary: one stream, no
    synchronisation in between, and the same again in a graph."""
    H, E, V = 256, 8, 500
    layer = Layer(E, 1, H, 384, MIX, seed=21)
    c, g = layer.ctx, layer.g
    qkv = [plain.make_page(c, block_weights(g, n, H), f) for n, f in ((256, "4"), (64, "8"), (64, "8"))]
    router = plain.make_page(c, block_weights(g, E, H), "16")
    vocabulary = plain.make_page(c, block_weights(g, V, H), "4")
    weight = (1 + 0.1 * normal(g, H)).half()
    stream0 = normal(g, T, H)
    attended = normal(g, T, H).half()              # stands in for an attention's output

    def step(residual):
        _, x, _, _ = c.pw_add_rmsnorm(attended, weight, 1e-6, residual=residual, residual_out=residual)
        three = c.pw_page_linear(x, qkv, out_features=[256, 64, 64])
        logits = c.pw_page_linear(x, [router], out_features=[E], out_dtype=F32)
        ids, gates = c.pw_route_tokens(logits, 2)
        y = c.pw_moe_forward_few_routed(0, x, ids, gates)
        _, z, _, _ = c.pw_add_rmsnorm(y, weight, 1e-6, residual=residual, residual_out=residual)
        return x, three, logits, ids, gates, y, z, c.pw_page_linear(z, [vocabulary], out_features=[V], out_dtype=F32)

    got = step(stream0.clone())
    torch.cuda.synchronize()
    x, three, logits, ids, gates, y, z, words = got
    parts = [plain.product(f64(x), [m[:n] for m in plain.stored(c, p)]) for n, p in zip((256, 64, 64), qkv)]
    check(three, np.concatenate([p[0] for p in parts], 1), np.concatenate([p[1] for p in parts], 1), F16)
    check(logits, *plain.product(f64(x), [m[:E] for m in plain.stored(c, router)]), F32)
    layer.check(y, x, [(t, e, float(gates[t, j])) for t, row in enumerate(ids.tolist()) for j, e in enumerate(row)])
    check(words, *plain.product(f64(z), [m[:V] for m in plain.stored(c, vocabulary)]), F32)
    residual = stream0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = step(residual)
    for _ in range(2):
        residual.copy_(stream0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, got))
    c.close()
