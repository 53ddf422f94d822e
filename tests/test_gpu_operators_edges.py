"""The operators around the layer on the GPU: memory handed over between warps and blocks, ends of the ranges, calls in
other orders and from other threads."""
import math
import threading
import time

import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2607_16184_b200 import binding as B
from paper_2607_16184_b200 import synth

from test_gpu_operators import F16, F32, BF16, U, check_linear, operands, randn
from util_gpu import build_layer, make_ctx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    yield c
    assert c.pw_last_device_status() == 0
    c.close()


@pytest.mark.parametrize("T", [5, 30, 50])
@pytest.mark.parametrize("tiles", [3, 14, 24, 34, 45, 70, 140])
def test_product_sums_of_clusters_again_and_again(ctx, T, tiles):
    """Every number of blocks that share a tile: sums and scales of one launch must not be those of the launch before."""
    K = 2100
    sets = [operands(ctx, T, tiles * 128 - 5, K, seed=7 * i) for i in range(3)]
    for s, f in zip(sets, (1.0, 64.0, 2.0 ** -9)):
        s[1].mul_(f)
    want = []
    for s in sets:
        out = torch.empty(T, tiles * 128 - 5, device="cuda")
        check_linear(ctx, *s, out)
        want.append(out)
    torch.cuda.synchronize()
    outs = [[torch.empty_like(want[0]) for _ in range(3)] for _ in range(2)]
    for i in range(90):
        ctx.pw_scaled_linear(*sets[i % 3], out=outs[i % 2][i % 3])
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for group in outs for o, w in zip(group, want))


@pytest.mark.parametrize("mode", [B.PW_MODE_SIMT, B.PW_MODE_TENSOR])
@pytest.mark.parametrize("T,n_experts", [(1, 16), (9, 64), (200, 16)])
def test_logits_of_a_product_directly_ahead_of_the_layer(T, n_experts, mode):
    """Router product -> pw_moe_forward, in one buffer of logits whose values change with every step."""
    cfg = synth.LayerConfig("ops_logits", n_experts, 4, 256, 384, T, n_shared=1, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x = synth.activations(cfg, device="cuda")
        q, qs = c.pw_quantize_scaled(x, 1)
        steps = []
        for i in range(4):
            w, sw = c.pw_quantize_scaled(randn(i, n_experts, 256, scale=0.2), 128)
            logits = c.pw_scaled_linear(q, qs, w, sw, out_dtype=F32)
            torch.cuda.synchronize()
            out = c.pw_moe_forward(0, x, logits, 4, mode=mode)
            torch.cuda.synchronize()
            ref = plain.route(logits, 4, "softmax", None, 1, 1, 1, True, 1.0)[0]
            assert np.array_equal(c.pw_get_routing(T, 4)["topk_ids"].cpu().numpy(), ref)
            steps.append((w, sw, out))
        logits = torch.empty(T, n_experts, device="cuda")
        got = [torch.empty_like(steps[0][2]) for _ in range(40)]
        for i in range(40):
            w, sw, _ = steps[i % 4]
            c.pw_scaled_linear(q, qs, w, sw, out=logits)
            c.pw_moe_forward(0, x, logits, 4, out=got[i], mode=mode)
        torch.cuda.synchronize()
        assert all(torch.equal(g, steps[i % 4][2]) for i, g in enumerate(got))
        assert not torch.equal(steps[0][2], steps[1][2]) and c.pw_last_device_status() == 0
    finally:
        c.close()


def test_other_threads_run_while_a_call_waits_for_the_queue(ctx):
    """A stream whose queue is full holds the call that launches, not the interpreter."""
    x, w = randn(1, 1, 256), randn(2, 256)
    y, s = torch.empty(1, 256, dtype=F16, device="cuda"), torch.cuda.Stream()
    ctx.pw_add_rmsnorm(x, w, y=y, stream=s)
    torch.cuda.synchronize()
    gap, stop = [0.0], threading.Event()

    def watch():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            gap[0], last = max(gap[0], now - last), now

    other = threading.Thread(target=watch)
    other.start()
    try:
        start = time.perf_counter()
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000_000)                 # about a second
        for _ in range(4000):
            ctx.pw_add_rmsnorm(x, w, y=y, stream=s)
        waited = time.perf_counter() - start
    finally:
        stop.set()
        other.join()
        torch.cuda.synchronize()
    assert gap[0] < max(0.25, 0.6 * waited), (gap[0], waited)    # it was all of the wait when the call kept the interpreter


def test_first_products_on_several_threads():
    """The first product of a context looks things up; four threads make it at the same time, and all launches count."""
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    try:
        sets = [operands(c, T, N, K, seed=T) for T, N, K in ((3, 2000, 1100), (40, 1000, 2100), (300, 500, 700), (1000, 520, 260))]
        before, outs, errors = c.pw_launch_count(), [[] for _ in sets], []
        torch.cuda.synchronize()
        ready = threading.Barrier(4)

        def work(i):
            try:
                s = torch.cuda.Stream()
                ready.wait()
                for _ in range(500):
                    outs[i] = outs[i][-3:] + [c.pw_scaled_linear(*sets[i], out_dtype=F32, stream=s)]
                s.synchronize()
            except Exception as e:                           # noqa: BLE001 - reported by the test
                errors.append(e)

        threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors and c.pw_launch_count() - before == 2000
        for i, (T, N) in enumerate(((3, 2000), (40, 1000), (300, 500), (1000, 520))):
            out = torch.empty(T, N, device="cuda")
            check_linear(c, *sets[i], out)
            assert all(torch.equal(o, out) for o in outs[i])
        assert c.pw_last_device_status() == 0
    finally:
        c.close()


SCALE_SHAPES = [(5, 300, 1400), (40, 390, 1300), (20, 20000, 390), (64, 19000, 260), (300, 500, 700), (1000, 512, 700), (2048, 4096, 390)]


def check_scales(ctx, a, sa, w, sw, out):
    """As check_linear, with the roundings of sums that are subnormal: one per block, half of 2^-149 each, and one when
    they are stored, which plain.rounding counts."""
    ctx.pw_scaled_linear(a, sa, w, sw, out=out)
    ref, mags = plain.linear(a, sa, w, sw)
    G = sa.shape[1]
    bound = mags * (4 * 2.0 ** -22 + (2 + G + 7) * U) + plain.rounding(ref, out.dtype) + (G + 7) * 2.0 ** -150
    got = plain.f64(out)
    assert np.isfinite(ref).all() and np.abs(ref).max() < 2.0 ** 127
    assert np.isfinite(got).all()
    assert np.all(np.abs(got - ref) <= bound * (1 + 4 * U)), float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max())
    return ref


@pytest.mark.parametrize("out_type", [F32, BF16])
@pytest.mark.parametrize("T,N,K", SCALE_SHAPES)
def test_product_of_scales_below_the_range(ctx, T, N, K, out_type):
    """Products of two scales that are subnormal or 0 in fp32, next to ordinary ones, while their sums are numbers."""
    a, sa, w, sw = operands(ctx, T, N, K, seed=T)
    rows = torch.tensor([0, -60, -80, -100, -118], device="cuda")[torch.arange(T, device="cuda") % 5]
    cols = torch.tensor([0, -20, -30, 10], device="cuda")[torch.arange(sw.shape[1], device="cuda") % 4]
    sa, sw = torch.ldexp(sa, rows[:, None]), torch.ldexp(sw, cols[None, :])
    f = plain.f64(sa)[:, :1] * plain.f64(sw)[:1, :]
    assert (f < 2.0 ** -126).any() and (f < 2.0 ** -149).any() and (f > 2.0 ** -100).any()
    ref = check_scales(ctx, a, sa, w, sw, torch.empty(T, N, dtype=out_type, device="cuda"))
    assert np.abs(ref).max() > 2.0 ** -20


def test_product_of_scales_the_quantizer_makes(ctx):
    """Activations near the smallest number that has a scale of its own, weights of ordinary size."""
    for T in (3, 1000):
        a, sa = ctx.pw_quantize_scaled(randn(1, T, 700, scale=2.0 ** -119), 1)
        w, sw = ctx.pw_quantize_scaled(randn(2, 600, 700, scale=0.01), 128)
        check_scales(ctx, a, sa, w, sw, torch.empty(T, 600, device="cuda"))


@pytest.mark.parametrize("out_type", [F32, BF16])
@pytest.mark.parametrize("T,N,K", SCALE_SHAPES)
def test_product_of_scales_above_the_range(ctx, T, N, K, out_type):
    """Products of two scales over the largest number: sums of the smallest codes are numbers, and sums of 0 are 0."""
    def small(rows, seed):
        q, s = B.scaled_empty(rows, K, 1)
        q.view(torch.uint8).copy_(torch.randint(0, 3, (rows, K), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda",
                                                dtype=torch.uint8))                 # 0, 2^-9, 2^-8
        q.view(torch.uint8)[::2] |= 0x80
        return q
    a, w = small(T, 1), small(N, 2)
    G = (K + 127) // 128
    sa = torch.ldexp(torch.ones(T, G, device="cuda"), torch.tensor([0, 60, 62, 100], device="cuda")[torch.arange(T, device="cuda") % 4][:, None])
    sw = torch.ldexp(torch.ones((N + 127) // 128, G, device="cuda"), torch.tensor([70, 10, 68], device="cuda")[torch.arange(G, device="cuda") % 3][None, :])
    a.view(torch.uint8)[3::4] = 0                                  # 2^100 * 2^70 times nothing
    check_scales(ctx, a, sa, w, sw, torch.empty(T, N, dtype=out_type, device="cuda"))


def test_product_of_scales_out_of_every_range(ctx):
    """What overflows is infinite, with the sign of the first block's sum (an fp32 sum that is infinite stays so, whatever
    finite product is added); what underflows is 0; a scale that is no number stays visible."""
    for T in (3, 1000):
        a, sa, w, sw = operands(ctx, T, 500, 200, seed=3)
        ref = plain.linear(a[:, :128], sa[:, :1], w[:, :128], sw[:, :1])[0]
        big = ctx.pw_scaled_linear(a, sa * 2.0 ** 110, w, sw * 2.0 ** 110, out_dtype=F32).cpu().numpy()
        assert np.array_equal(big, np.where(ref > 0, np.inf, -np.inf))
        none = ctx.pw_scaled_linear(a, torch.ldexp(sa, torch.tensor(-110, device="cuda")), w, torch.ldexp(sw, torch.tensor(-110, device="cuda")), out_dtype=F32)
        assert bool((none == 0).all())
        bad = sa.clone()
        bad[1], bad[2, 1] = math.inf, math.nan
        out = ctx.pw_scaled_linear(a, bad, w, sw, out_dtype=F32).cpu().numpy()
        assert not np.isfinite(out[1:3]).any() and np.isnan(out[2]).all() and np.isfinite(out[0]).all()


@pytest.mark.parametrize("cols", [1, 300, 264])
def test_single_rows_of_codes_as_they_lie(ctx, cols):
    """One row needs no stride: contiguous codes of a width that is no multiple of 16, and a stride that is one of nothing."""
    x, w, r = randn(1, 1, cols), randn(2, cols), randn(3, 1, cols)
    for q in (torch.empty(1, cols, dtype=torch.uint8, device="cuda"), torch.empty(5000, dtype=torch.uint8, device="cuda").as_strided((1, cols), (1237, 1))):
        want, scales = ctx.pw_quantize_scaled(x, 1)
        _, s = ctx.pw_quantize_scaled(x, 1, q=q, scales=torch.empty_like(scales))
        assert torch.equal(q, want.view(torch.uint8)) and torch.equal(s, scales)
        want, scales = B.scaled_empty(1, cols, 1)
        ctx.pw_add_rmsnorm(x, w, residual=r, q=want, q_scales=scales)
        _, _, _, s = ctx.pw_add_rmsnorm(x, w, residual=r, q=q, q_scales=torch.empty_like(scales))
        assert torch.equal(q, want.view(torch.uint8)) and torch.equal(s, scales)
        many, ms = ctx.pw_quantize_scaled(randn(4, 200, cols), 128)
        out = torch.empty(1, 200, device="cuda")
        check_linear(ctx, q.view(torch.float8_e4m3fn), s, many, ms, out)
        assert torch.equal(out, ctx.pw_scaled_linear(want, scales, many, ms, out_dtype=F32))
        one, os = ctx.pw_quantize_scaled(x, 128, q=q, scales=torch.empty_like(scales))
        for T in (1, 70, 1000):
            a, sa = ctx.pw_quantize_scaled(randn(5, T, cols), 1)
            check_linear(ctx, a, sa, one.view(torch.float8_e4m3fn), os, torch.empty(T, 1, device="cuda"))


def test_arguments_that_do_not_fit_are_refused_and_nothing_runs(ctx):
    """Integers beyond 32 bits are not cut to others; what is no number at all raises before anything is launched."""
    x, big = randn(1, 1, 256), 1 << 32
    q, s = B.scaled_empty(1, 256, 1)
    ids, gates = torch.full((1, 2), 7, dtype=torch.int32, device="cuda"), torch.full((1, 2), 7.0, device="cuda")
    hidden = torch.zeros(1, 256, dtype=F16, device="cuda")
    torch.cuda.synchronize()
    before = ctx.pw_launch_count()
    route = lambda **kw: ctx.pw_route_tokens(x, **{**dict(top_k=2, ids=ids, gates=gates), **kw})
    for call in (lambda: ctx.pw_quantize_scaled(x, big + 1, q=q, scales=s), lambda: route(top_k=big + 2), lambda: route(top_k=-big + 2),
                 lambda: route(n_groups=big + 1), lambda: route(top_groups=big + 1), lambda: route(group_best=(1 << 70) + 1), lambda: route(scale=1e300),
                 lambda: ctx.pw_moe_forward_routed(big, hidden, ids, gates), lambda: ctx.pw_moe_forward_routed(0, hidden, ids, gates, mode=big)):
        with pytest.raises(B.PwError) as e:
            call()
        assert e.value.status == 1, str(e.value)
    for call in (lambda: ctx.pw_quantize_scaled(x, 1.0, q=q, scales=s), lambda: route(scale=None), lambda: route(scale="1"), lambda: route(n_groups=1.0),
                 lambda: ctx.pw_add_rmsnorm(x, x[0], eps=None, y=torch.empty_like(x)), lambda: ctx.pw_moe_forward_routed("0", hidden, ids, gates)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(RuntimeError):
        route(renormalize=torch.zeros(2))
    torch.cuda.synchronize()
    assert ctx.pw_launch_count() == before and bool((ids == 7).all()) and bool((gates == 7).all())


def test_context_keeps_the_device_it_was_made_on(ctx):
    """A context of "cuda" belongs to one device, on which its outputs are made whatever device is current later."""
    assert ctx.device == torch.device("cuda", torch.cuda.current_device())
    assert ctx.pw_quantize_scaled(randn(1, 2, 128), 1)[0].device == ctx.device == ctx.workspace.device


@pytest.mark.parametrize("T,n_experts", [(4, 16), (4, 64), (4, 200), (300, 16)])
def test_layer_of_logits_that_are_no_numbers(T, n_experts):
    """Rows with fewer numbers than choices: distinct experts, gate 0 for those without a number, other rows as they were."""
    cfg = synth.LayerConfig("ops_nan", n_experts, 4, 256, 384, T, n_shared=1, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x = synth.activations(cfg, device="cuda")
        logits = randn(1, T, n_experts)
        want = c.pw_moe_forward(0, x, logits, 4).clone()
        bad = logits.clone()
        bad[0] = math.nan
        bad[1] = math.nan
        bad[1, 5], bad[1, 11] = 0.5, -0.5
        bad[2, ::2] = math.nan
        got = c.pw_moe_forward(0, x, bad, 4)
        r = {n: v.cpu().numpy() for n, v in c.pw_get_routing(T, 4).items()}
        ids, gates = r["topk_ids"], r["gates"]
        assert ids.min() >= 0 and ids.max() < n_experts and all(len(set(row)) == 4 for row in ids)
        assert np.array_equal(np.sort(r["perm"]), np.arange(T * 4)) and r["counts"].sum() == T * 4
        assert list(ids[0]) == [0, 1, 2, 3] and np.isnan(gates[0]).all()
        assert list(ids[1]) == [5, 11, 0, 1] and np.allclose(gates[1], [1 / (1 + math.exp(-1)), 1 - 1 / (1 + math.exp(-1)), 0, 0])
        assert (ids[2] % 2 == 1).all()
        got, want = got.cpu().numpy(), want.cpu().numpy()
        assert np.isnan(got[0]).all() and np.isfinite(got[1:]).all()
        near = np.abs(got[3:] - want[3:])
        assert near.max() <= 2e-2                              # other neighbours in their tiles, so other orders of sums
        static = B.pw_route_tokens_static(bad, 4)
        assert np.array_equal(static["topk_ids"].cpu().numpy(), ids)
        assert c.pw_last_device_status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(72, 6), (128, 8), (160, 6), (256, 8), (256, 31), (250, 1), (100, 32)])
def test_router_near_ties_with_a_bias_and_no_groups(ctx, score, E, k):
    """Keys that 32 bits cannot tell apart among more than 64 experts: logits one step apart under the same bias, runs of
    such logits at the cut, equal ones, and biases that give back what the scores differ by."""
    T = 160
    g = torch.Generator().manual_seed(E + k)
    x = torch.randn(T, E, generator=g) * 0.5
    bias = torch.randn(E, generator=g) * 0.05
    bias[1::2] = bias[: E // 2 * 2: 2]
    x[:, 1::2] = torch.nextafter(x[:, : E // 2 * 2: 2], torch.full((T, E // 2), math.inf))
    x[::3, 1::2] = x[::3, : E // 2 * 2: 2]                        # equal in everything
    # runs of 3, 12 and 40 experts on one logit and one bias, moved by up to two steps, from the best on
    for row, n in ((1, 3), (4, 12), (7, 40), (10, 3), (13, 12), (16, 40)):
        x[row, : n] = 2.0
        for _ in range(2):
            move = torch.rand(n, generator=g) < 0.5
            x[row, :n] = torch.where(move, torch.nextafter(x[row, :n], torch.full((n,), math.inf)), x[row, :n])
    bias[: 40] = bias[0]
    # a row whose keys are all alike up to the rounding of the bias
    far = plain.f64(x[20])
    p = 1 / (1 + np.exp(-far)) if score == "sigmoid" else np.exp(far - far.max()) / np.exp(far - far.max()).sum()
    flat = torch.from_numpy((0.5 - p).astype(np.float32))
    for b in (bias, flat):
        logits = x.cuda()
        ids, gates = ctx.pw_route_tokens(logits, k, score=score, bias=b.cuda())
        ref_ids, ref_gates = plain.route(logits, k, score, plain.f64(b), 1, 1, 1, True, 1.0)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        np.testing.assert_allclose(gates.cpu().numpy(), ref_gates, rtol=52 * U)


def test_first_product_of_a_context_inside_a_capture():
    """What the first product looks up is no work on the stream: it may happen while one is captured."""
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    try:
        shapes = [(3, 700, 1100), (40, 1000, 2100), (300, 500, 700), (1000, 2048, 512)]
        sets = [operands(c, T, N, K, seed=T) for T, N, K in shapes]
        outs = [torch.full((T, N), 5.0, device="cuda") for T, N, _ in shapes]
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for ops, out in zip(sets, outs):
                c.pw_scaled_linear(*ops, out=out, stream=s)
        torch.cuda.synchronize()
        assert all(bool((o == 5).all()) for o in outs)                 # captured, not run
        g.replay()
        torch.cuda.synchronize()
        for ops, out in zip(sets, outs):
            want = torch.empty_like(out)
            check_linear(c, *ops, want)
            assert torch.equal(out, want)
        assert c.pw_last_device_status() == 0
        del g
    finally:
        c.close()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_codes_are_those_of_the_quotient_but_next_to_a_middle(ctx, block_rows):
    """A code is within half a step of value / scale, and of two fp32 roundings (reciprocal, product) of the quotient."""
    x = randn(block_rows, 300, 1000) * torch.exp(randn(2, 300, 1) * 3)
    q, s = ctx.pw_quantize_scaled(x, block_rows)
    v = plain.f64(x) / plain.spread(plain.f64(s), block_rows, x.shape)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -30))), -6) - 3)
    assert np.all(np.abs(plain.code_values(q) - v) <= step / 2 + np.abs(v) * 2 * U * (1 + U))


@pytest.mark.parametrize("n_groups", [1, 4])
@pytest.mark.parametrize("E", [16, 64, 128])
def test_router_biases_that_are_no_numbers(ctx, E, n_groups):
    """NaN and -infinity close an expert, +infinity takes it first; the gates are those of the scores alone."""
    T, k = 40, 6
    x = randn(E, T, E)
    bias = randn(E + 1, E, scale=0.1)
    bias[E // 2] = math.inf
    bias[:3], bias[3] = math.nan, -math.inf
    few = torch.full_like(bias, -math.inf)
    few[5], few[E - 1] = 0.0, 1.0
    for b, open_ in ((bias, None), (few, {5, E - 1})):
        ids, gates = ctx.pw_route_tokens(x, k, score="sigmoid", bias=b, n_groups=n_groups, top_groups=2 if n_groups > 1 else 1, renormalize=False)
        i, g = ids.cpu().numpy(), plain.f64(gates)
        if open_ is None:
            assert i.min() >= 4 and (i[:, 0] == E // 2).all() and all(len(set(r)) == k for r in i)
        else:
            assert all(set(r) == open_ | {-1} and list(r[2:]) == [-1] * 4 and r[0] == E - 1 for r in i)
        p = 1 / (1 + np.exp(-plain.f64(x)))
        want = np.where(i >= 0, np.take_along_axis(p, np.maximum(i, 0), 1), 0.0)
        assert np.all(np.abs(g - want) <= want * 52 * U)


def test_norm_at_the_ends_of_the_range(ctx):
    """Squares over fp32's range give 0, squares under it count as 0; the row of the residual is what it is."""
    x = torch.zeros(4, 256, device="cuda")
    x[0], x[1], x[2, 0] = 2.0 ** 64, 2.0 ** -76, 2.0 ** 62
    w, r = torch.ones(256, device="cuda"), torch.zeros(4, 256, device="cuda")
    ro, y = torch.empty_like(x), torch.empty_like(x)
    ctx.pw_add_rmsnorm(x, w, 1e-6, residual=r, residual_out=ro, y=y)
    assert torch.equal(ro, x) and bool((y[0] == 0).all()) and bool((y[3] == 0).all())
    assert abs(float(y[2, 0]) - 16.0) <= 16 * 43 * U and abs(float(y[1, 0]) * 2.0 ** 76 / 1e3 - 1) <= 43 * U + 1e-6
    ctx.pw_add_rmsnorm(x, w, 0.0, y=y)
    assert bool(torch.isnan(y[3]).all()) and not bool(torch.isfinite(y[1]).any())


@pytest.mark.parametrize("T,H,pad", [(3, 520, 0), (3, 521, 2), (200, 4096, 0), (2, 20001, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_outputs_over_its_inputs(ctx, T, H, pad, dtype):
    """Every overlap that the header allows gives what separate buffers give."""
    def buffer(seed):
        whole = torch.zeros(T, H + pad, dtype=dtype, device="cuda")
        whole[:, :H] = randn(seed, T, H)
        return whole[:, :H]

    w = randn(3, H)
    x, r, ro, y = buffer(1), buffer(2), torch.zeros(T, H + pad, dtype=dtype, device="cuda")[:, :H], torch.zeros(T, H + pad, dtype=dtype, device="cuda")[:, :H]
    q, qs = B.scaled_empty(T, H, 1)
    ctx.pw_add_rmsnorm(x, w, residual=r, residual_out=ro, y=y, q=q, q_scales=qs)
    for where_ro, where_y in (("x", None), ("r", None), ("r", "x"), ("x", "r"), (None, "x"), (None, "r"), ("x", "x"), ("r", "r"), ("new", "new")):
        b = {"x": buffer(1), "r": buffer(2), "new": torch.zeros(T, H + pad, dtype=dtype, device="cuda")[:, :H]}
        out = torch.zeros(T, H + pad, dtype=dtype, device="cuda")[:, :H] if where_y is None else b[where_y]
        q2, qs2 = B.scaled_empty(T, H, 1)
        ctx.pw_add_rmsnorm(b["x"], w, residual=b["r"], residual_out=None if where_ro is None else b[where_ro], y=out, q=q2, q_scales=qs2)
        assert torch.equal(out, y) and torch.equal(qs2, qs) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8))
        if where_ro is not None and where_ro != where_y:
            assert torch.equal(b[where_ro], ro)


def test_layer_and_operators_on_two_streams_at_once(ctx):
    """A layer on one stream, the operators around another one on a second: neither changes what the other computes."""
    cfg = synth.LayerConfig("ops_beside", 16, 4, 512, 1024, 64, n_shared=1, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x, logits = synth.activations(cfg, device="cuda"), synth.router_logits(cfg, device="cuda")
        sets = [operands(ctx, T, N, K, seed=T) for T, N, K in ((5, 4096, 2048), (64, 3000, 2048), (300, 1000, 1024), (1500, 2048, 1024))]
        rows, w = randn(1, 700, 2056), randn(2, 2056)
        wide = randn(3, 900, 256)

        def around(s=None):
            return [ctx.pw_scaled_linear(*ops, out_dtype=F32, stream=s) for ops in sets] + [ctx.pw_add_rmsnorm(rows, w, stream=s)[1]] + \
                list(ctx.pw_route_tokens(wide, 8, score="sigmoid", bias=wide[0], n_groups=8, top_groups=4, group_best=2, stream=s)) + \
                list(ctx.pw_quantize_scaled(rows, 128, stream=s))

        def layer(s=None):
            ids, gates = c.pw_route_tokens(logits, 4, stream=s)
            return [c.pw_moe_forward(0, x, logits, 4, stream=s), c.pw_moe_forward_routed(0, x, ids, gates, stream=s)]

        want_a, want_l = around(), layer()
        torch.cuda.synchronize()
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        got_a, got_l = [], []
        for _ in range(15):
            with torch.cuda.stream(b):
                got_l.append(layer(b))
            with torch.cuda.stream(a):
                got_a.append(around(a))
        torch.cuda.synchronize()
        bits = lambda t: t.contiguous().view(torch.uint8)
        for want, runs in ((want_a, got_a), (want_l, got_l)):
            for got in runs:
                assert all(torch.equal(bits(g), bits(v)) for g, v in zip(got, want))
        assert c.pw_last_device_status() == 0 and ctx.pw_last_device_status() == 0
    finally:
        c.close()
