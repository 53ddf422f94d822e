"""The operators around the layer on the GPU against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2607_16184_b200 import binding as B
from paper_2607_16184_b200 import synth

from util_gpu import build_layer, error_metrics, export_to_oracle, make_ctx

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = 2.0 ** -24                                     # half a step of fp32


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    yield c
    assert c.pw_last_device_status() == 0
    c.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen(seed), device="cuda") * scale).to(dtype)


def strided(rows, cols, pad, dtype, fill=0.0):
    """A view [rows, cols] with `pad` more columns between rows and two more rows behind; and the whole buffer."""
    whole = torch.full((rows + 2, cols + pad), fill, device="cuda").to(dtype)
    return whole[:rows, :cols], whole


def guards_left(whole, view, fill):
    keep = torch.ones_like(whole, dtype=torch.bool)
    keep[:view.shape[0], :view.shape[1]] = False
    return bool((whole[keep].float() == torch.tensor(fill).to(whole.dtype).float()).all())


# ---- quantizer -------------------------------------------------------------------------------------

@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (3, 127, 1), (5, 129, 7), (130, 264, 8), (257, 520, 0), (33, 1408, 16), (300, 2055, 3), (67, 1001, 0),
                                           (40, 2047, 0), (9, 1025, 2), (200, 3, 0), (150, 1, 0), (131, 5, 1), (140, 1023, 4)])
def test_quantizer_bit_for_bit(ctx, rows, cols, pad, dtype, block_rows):
    x, _ = strided(rows, cols, pad, dtype)
    x.copy_(randn(rows * cols, rows, cols))
    x[0, :min(cols, 128)] = 0                                       # a block of zeros (block_rows 1)
    whole = torch.full((rows + 2, (cols + 15) // 16 * 16 + 16), 0x5a, dtype=torch.uint8, device="cuda")
    q = whole[:rows, :cols]
    scales = B.scaled_empty(rows, cols, block_rows)[1]
    ctx.pw_quantize_scaled(x, block_rows, q=q, scales=scales)
    codes, ref = plain.quantize_bits(x, block_rows)
    assert np.array_equal(scales.cpu().numpy(), ref)
    # -0 and +0 are the same value; everything else is compared bit for bit
    got = q.cpu().numpy().copy()
    got[got == 0x80], codes[codes == 0x80] = 0, 0
    assert np.array_equal(got, codes)
    whole[:rows, :cols] = 0x5a
    assert bool((whole == 0x5a).all())


def test_quantizer_of_extreme_values(ctx):
    x = torch.zeros(6, 256, device="cuda")
    x[0], x[1, ::2], x[2], x[3] = 3.0e38, 1e-38, 1e-45, -448.0
    x[4] = torch.linspace(-1, 1, 256, device="cuda") * 2.0 ** -130
    q, s = ctx.pw_quantize_scaled(x, 1)
    codes, ref = plain.quantize_bits(x, 1)
    assert np.array_equal(s.cpu().numpy(), ref) and np.isfinite(ref).all()
    assert np.array_equal(plain.code_values(q), plain.code_values(torch.from_numpy(codes)))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cols", [256, 131])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_of_infinities_and_nan(ctx, cols, dtype, block_rows):
    x = randn(cols, 140, cols, dtype=dtype)
    x[0, 3], x[1, 7], x[130, 130] = math.nan, -math.inf, math.inf
    x[131] = math.nan
    x[139, 128:] = math.nan
    q, s = ctx.pw_quantize_scaled(x, block_rows)
    # scales of the numbers that are none left out; infinite where an infinity is in the block
    clean = torch.where(x.isfinite(), x, torch.zeros_like(x))
    codes, ref = plain.quantize_bits(clean, block_rows)
    inf = plain.block_tops(x.isinf().double().cpu().numpy(), block_rows) > 0
    assert inf.sum() == 2
    ref[inf] = np.inf
    assert np.array_equal(s.cpu().numpy(), ref)
    want = plain.code_values(torch.from_numpy(codes))
    want[plain.spread(inf, block_rows, want.shape)] = 0
    want[~x.isfinite().cpu().numpy()] = np.nan
    assert np.array_equal(plain.code_values(q), want, equal_nan=True)


# ---- norm ------------------------------------------------------------------------------------------

# Relative error of y before its rounding: one rounding of s; the sum of squares is a chain of at most 64 fused
# additions per thread and 10 across threads, the division, eps, root and reciprocal one each, of which the root halves
# what came before it: (64 + 10 + 2) / 2 + 2; two products.  43 roundings.
NORM_REL = 43 * U


def check_norm(x, residual, w, eps, residual_out, y, q, q_scales):
    s, ref = plain.rmsnorm(x, residual, w, eps)
    if residual_out is not None:
        assert np.all(np.abs(plain.f64(residual_out) - s) <= plain.rounding(s, residual_out.dtype) * (1 + 2 * U) + np.abs(s) * U)
    if y is not None:
        assert np.all(np.abs(plain.f64(y) - ref) <= (plain.rounding(ref, y.dtype) + np.abs(ref) * NORM_REL) * (1 + 2 * U))
    if q is not None:
        tops = plain.block_tops(ref, 1)
        scales = np.where(tops == 0, 1.0, np.maximum(tops / 448, 2.0 ** -126))
        got = plain.f64(q_scales)
        assert np.all(np.abs(got - scales) <= scales * (NORM_REL + 2 * U))
        # a code is half a step off at most: 2^-4 of the value, half of 2^-9 scales below the smallest normal code;
        # reciprocal and product round once each
        per = plain.spread(got, 1, ref.shape)
        bound = np.maximum(np.abs(ref) * 2.0 ** -4, per * 2.0 ** -10) + np.abs(ref) * (2 * NORM_REL + 8 * U)
        assert np.all(np.abs(plain.code_values(q) * per - ref) <= bound)


@pytest.mark.parametrize("x_type,res_type,w_type,y_type", [(F32, F16, F16, F16), (F16, F16, F16, F16), (BF16, BF16, BF16, BF16), (F32, F32, F32, F32),
                                                          (F32, BF16, F32, F16), (F16, None, BF16, BF16), (BF16, F32, F16, F32), (F32, None, F32, F16),
                                                          (F16, BF16, F32, None), (BF16, F16, BF16, F32), (BF16, None, BF16, F16), (F16, F32, F16, BF16)])
@pytest.mark.parametrize("T,H,pad", [(1, 1, 0), (2, 7, 1), (3, 128, 0), (5, 257, 0), (4, 4096, 8), (3, 2056, 0), (2, 4104, 3), (2, 8184, 0), (2, 9001, 0), (1, 16392, 0)])
def test_norm_types_and_widths(ctx, T, H, pad, x_type, res_type, w_type, y_type):
    x, _ = strided(T, H, pad, x_type)
    x.copy_(randn(H, T, H))
    w = (1 + randn(H + 1, H, scale=0.2)).to(w_type)
    residual = ro = None
    if res_type is not None:
        residual, _ = strided(T, H, pad, res_type)
        residual.copy_(randn(H + 2, T, H, scale=3.0))
        ro, ro_whole = strided(T, H, pad, res_type, 7.0)
    y = None
    if y_type is not None:
        y, y_whole = strided(T, H, pad, y_type, 7.0)
    q, qs = B.scaled_empty(T, H, 1)
    ctx.pw_add_rmsnorm(x, w, 1e-6, residual=residual, residual_out=ro, y=y, q=q, q_scales=qs)
    check_norm(x, residual, w, 1e-6, ro, y, q, qs)
    if ro is not None:
        assert guards_left(ro_whole, ro, 7.0)
    if y is not None:
        assert guards_left(y_whole, y, 7.0)


@pytest.mark.parametrize("T", [100, 300])
@pytest.mark.parametrize("H", [5120, 8191, 9728, 9729, 16384, 20000])
def test_norm_of_fewer_and_more_rows_than_sms(ctx, T, H):
    x, w, r = randn(1, T, H, dtype=BF16), randn(2, H), randn(3, T, H)
    y, ro = torch.empty(T, H, dtype=BF16, device="cuda"), torch.empty_like(r)
    q, qs = B.scaled_empty(T, H, 1)
    ctx.pw_add_rmsnorm(x, w, 1e-5, residual=r, residual_out=ro, y=y, q=q, q_scales=qs)
    check_norm(x, r, w, 1e-5, ro, y, q, qs)


@pytest.mark.parametrize("H", [24573, 32768])
def test_norm_of_the_widest_rows(ctx, H):
    x, w, r = randn(1, 2, H), randn(2, H), randn(3, 2, H, dtype=F16)
    y, ro = torch.empty(2, H, dtype=F32, device="cuda"), torch.empty_like(r)
    q, qs = B.scaled_empty(2, H, 1)
    ctx.pw_add_rmsnorm(x, w, 1e-5, residual=r, residual_out=ro, y=y, q=q, q_scales=qs)
    check_norm(x, r, w, 1e-5, ro, y, q, qs)
    with pytest.raises(B.PwError) as e:
        ctx.pw_add_rmsnorm(torch.zeros(1, 32769, device="cuda"), torch.zeros(32769, device="cuda"))
    assert e.value.status == 2


def test_norm_in_place_and_row_of_zeros(ctx):
    T, H = 33, 520
    x, r, w = randn(1, T, H, dtype=F16), randn(2, T, H, dtype=F16), randn(3, H, dtype=F16)
    x[5], r[5] = 0, 0
    want = [t.clone() for t in ctx.pw_add_rmsnorm(x, w, 1e-6, residual=r, residual_out=torch.empty_like(r), y=torch.empty_like(x))[:2]]
    xi, ri = x.clone(), r.clone()
    ctx.pw_add_rmsnorm(xi, w, 1e-6, residual=ri, residual_out=ri, y=xi)       # residual and x written over
    assert torch.equal(ri, want[0]) and torch.equal(xi, want[1])
    assert bool((want[1][5] == 0).all())
    q, qs = B.scaled_empty(T, H, 1)
    ctx.pw_add_rmsnorm(x, w, 1e-6, residual=r, q=q, q_scales=qs)
    assert bool((qs[5] == 1).all()) and bool((q[5].float() == 0).all())


def test_rows_far_apart(ctx):
    """Element offsets past 32 bits: rows 2^31 + 64 elements apart."""
    H, pitch = 264, (1 << 31) + 64
    whole = torch.empty(2 * pitch + H, dtype=F16, device="cuda")
    x = whole.as_strided((3, H), (pitch, 1))
    x.copy_(randn(4, 3, H))
    w = randn(5, H)
    y = torch.empty(3, H, dtype=F32, device="cuda")
    q, qs = B.scaled_empty(3, H, 1)
    ctx.pw_add_rmsnorm(x, w, 1e-6, y=y, q=q, q_scales=qs)
    check_norm(x, None, w, 1e-6, None, y, q, qs)
    q, qs = ctx.pw_quantize_scaled(x, 128)
    codes, ref = plain.quantize_bits(x, 128)
    assert np.array_equal(qs.cpu().numpy(), ref) and np.array_equal(plain.code_values(q), plain.code_values(torch.from_numpy(codes)))
    out = whole.as_strided((3, 200), (pitch, 1))
    a, sa = ctx.pw_quantize_scaled(randn(6, 3, 300), 1)
    b, sb = ctx.pw_quantize_scaled(randn(7, 200, 300), 128)
    check_linear(ctx, a, sa, b, sb, out)


# ---- product ---------------------------------------------------------------------------------------

def check_linear(ctx, a, sa, w, sw, out):
    ctx.pw_scaled_linear(a, sa, w, sw, out=out)
    ref, mags = plain.linear(a, sa, w, sw)
    G = sa.shape[1]
    # Products of two codes are exact in fp32.  A block is four tensor-core steps; what one adds is taken to be cut, not
    # rounded, after aligning, at 2^-22 of the magnitudes added so far.  Then per block one product of the scales, one
    # fused multiply-add, and up to three additions between the ranges that share a tile.
    bound = mags * (4 * 2.0 ** -22 + (2 + G + 7) * U) + plain.rounding(ref, out.dtype)
    err = np.abs(plain.f64(out) - ref)
    assert np.all(err <= bound * (1 + 4 * U)), (float((err / np.maximum(bound, 1e-300)).max()), tuple(out.shape), w.shape)


def operands(ctx, T, N, K, seed=0, pad=0):
    def codes(rows, scale, block, s):
        q, sc = B.scaled_empty(rows, K + pad, block)
        q = q[:, :K]
        sc = torch.empty(sc.shape[0], (K + 127) // 128, device="cuda")
        return ctx.pw_quantize_scaled(randn(s, rows, K, scale=scale), block, q=q, scales=sc)
    return (*codes(T, 1.0, 1, seed + 1), *codes(N, 0.02, 128, seed + 2))


@pytest.mark.parametrize("out_type", [F32, F16, BF16])
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (1, 8, 16), (1, 128, 128), (2, 129, 127), (7, 64, 2056), (16, 130, 384), (17, 256, 1000), (33, 200, 2048),
                                   (64, 384, 640), (65, 127, 500), (128, 128, 4096), (129, 257, 300), (301, 64, 2056), (300, 1000, 1408),
                                   (1030, 520, 700), (2048, 4100, 512), (1500, 4099, 300)])
def test_product_sizes_and_types(ctx, T, N, K, out_type):
    a, sa, w, sw = operands(ctx, T, N, K, seed=T + N + K)
    out, whole = strided(T, N, 5, out_type, 7.0)
    check_linear(ctx, a, sa, w, sw, out)
    assert guards_left(whole, out, 7.0)


@pytest.mark.parametrize("out_type", [F32, F16, BF16])
@pytest.mark.parametrize("T,N,K,pad", [(70, 127, 500, 1), (200, 130, 129, 6), (200, 132, 300, 4), (300, 264, 700, 8), (300, 520, 256, 24), (129, 1032, 256, 16),
                                       (2000, 4104, 256, 8), (2000, 4108, 256, 4), (1999, 4097, 256, 7)])
def test_product_leaves_what_lies_between_rows(ctx, T, N, K, pad, out_type):
    """Rows a multiple of 16 bytes apart, whose length may or may not be one."""
    a, sa, w, sw = operands(ctx, T, N, K, seed=T + N + K)
    out, whole = strided(T, N, pad, out_type, 7.0)
    check_linear(ctx, a, sa, w, sw, out)
    assert guards_left(whole, out, 7.0)


@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (64, 2048, 14336), (48, 5244, 2607), (16, 4999, 1300), (3, 3700, 700), (30, 3200, 1290), (64, 3300, 1290),
                                   (64, 20000, 260), (13, 30000, 130), (256, 4096, 1408), (512, 1500, 2048), (1000, 2048, 1024), (1030, 770, 391), (2048, 4096, 512)])
def test_product_larger(ctx, T, N, K):
    a, sa, w, sw = operands(ctx, T, N, K, seed=T, pad=32)
    check_linear(ctx, a, sa, w, sw, torch.empty(T, N, dtype=F16, device="cuda"))


def test_product_of_uneven_scales(ctx):
    """Scales over twelve orders of magnitude, per row and per block: an error of one scale's place shows."""
    T, N, K = 70, 300, 700
    x = randn(1, T, K) * torch.logspace(-6, 6, T, device="cuda")[:, None]
    y = randn(2, N, K) * torch.logspace(3, -3, K, device="cuda")[None, :]
    y[128:256] *= 1e4
    a, sa = ctx.pw_quantize_scaled(x, 1)
    w, sw = ctx.pw_quantize_scaled(y, 128)
    check_linear(ctx, a, sa, w, sw, torch.empty(T, N, dtype=F32, device="cuda"))


def test_product_gives_the_same_bits_again(ctx):
    for T, N, K in ((3, 4096, 4096), (64, 1408, 2048), (700, 2048, 1408)):
        a, sa, w, sw = operands(ctx, T, N, K)
        first = ctx.pw_scaled_linear(a, sa, w, sw, out_dtype=F32)
        for _ in range(5):
            assert torch.equal(first, ctx.pw_scaled_linear(a, sa, w, sw, out_dtype=F32))


def test_products_on_two_streams_at_once(ctx):
    """No call keeps anything that another one uses."""
    shapes = [(40, 4096, 1400), (300, 1000, 900), (5, 5000, 700), (64, 2048, 2048), (1000, 600, 512), (20, 20000, 260)]
    sets = [operands(ctx, *s, seed=i) for i, s in enumerate(shapes)]
    want = [ctx.pw_scaled_linear(*s, out_dtype=F32) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[torch.empty_like(w) for w in want] for _ in range(2)]
    for n in range(20):
        for k, st in enumerate(streams):
            for i in range(len(sets)):
                j = (i + 3 * k + n) % len(sets)
                ctx.pw_scaled_linear(*sets[j], out=got[k][j], stream=st)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want, got[k]))
    assert ctx.pw_last_device_status() == 0


@pytest.mark.parametrize("T", [1, 20, 40, 64, 300])
def test_product_back_to_back(ctx, T):
    """Long contractions from HBM, launch after launch: copies land out of order, stages and barriers are used many times."""
    N, K = 4096, 14336
    sets = [operands(ctx, T, N, K, seed=100 * i) for i in range(3)]
    want = [ctx.pw_scaled_linear(*s, out_dtype=F32) for s in sets]
    torch.cuda.synchronize()
    outs = [[torch.empty_like(want[0]) for _ in range(3)] for _ in range(2)]
    for i in range(60):
        ctx.pw_scaled_linear(*sets[i % 3], out=outs[i % 2][i % 3])
    torch.cuda.synchronize()
    assert ctx.pw_last_device_status() == 0
    for group in outs:
        assert all(torch.equal(o, w) for o, w in zip(group, want))


def test_product_wait_that_runs_out_is_reported():
    c = B.Context(1, 8, 0, 256, 512, 16, 2)
    try:
        for T, N, K in ((5, 300, 14336), (40, 300, 4096), (1000, 512, 1024)):
            a, sa, w, sw = operands(c, T, N, K)
            c.pw_debug_set_wait(1, 2)
            c.pw_scaled_linear(a, sa, w, sw)
            assert c.pw_last_device_status() == 8
            c.pw_debug_set_wait()
            check_linear(c, a, sa, w, sw, torch.empty(T, N, dtype=F16, device="cuda"))
            assert c.pw_last_device_status() == 0
    finally:
        c.close()


# ---- router ----------------------------------------------------------------------------------------

RULES = [dict(E=8, k=2), dict(E=1, k=1), dict(E=33, k=32), dict(E=64, k=6, renormalize=False), dict(E=60, k=4, score="sigmoid"),
         dict(E=128, k=8, score="sigmoid", bias=True, scale=2.5), dict(E=256, k=8, score="sigmoid", bias=True, n_groups=8, top_groups=4, group_best=2, scale=2.5),
         dict(E=256, k=8, n_groups=8, top_groups=3, group_best=1), dict(E=160, k=6, n_groups=8, top_groups=3, group_best=1, renormalize=False, scale=16.0),
         dict(E=96, k=5, n_groups=3, top_groups=2, group_best=2, renormalize=False), dict(E=64, k=3, n_groups=64, top_groups=5, group_best=2, bias=True),
         dict(E=200, k=32, n_groups=2, top_groups=2, group_best=2), dict(E=256, k=32, bias=True)]


def check_route(ctx, logits, rule):
    rule = dict(rule)
    E, k = rule.pop("E"), rule.pop("k")
    bias = randn(E, E, scale=0.1) if rule.pop("bias", False) else None
    args = dict(score="softmax", n_groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0)
    args.update(rule)
    ids, gates = ctx.pw_route_tokens(logits, k, bias=bias, **args)
    ref_ids, ref_gates = plain.route(logits, k, bias=None if bias is None else plain.f64(bias), **args)
    assert np.array_equal(ids.cpu().numpy(), ref_ids)
    # one rounding; without renormalisation the softmax's denominator is a sum in fp32 of at most 8 + 5 additions of
    # exponentials that are two steps (four half steps) and one rounded difference off (|l - top| < 2^5 here: 32 half steps)
    got = plain.f64(gates)
    assert np.all(np.abs(got - ref_gates) <= ref_gates * 52 * U + 2.0 ** -149)


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("dtype,T,pad", [(F32, 1, 0), (F32, 131, 3), (BF16, 67, 0), (F16, 5, 1)])
def test_router_rules(ctx, rule, dtype, T, pad):
    logits, _ = strided(T, rule["E"], pad, dtype)
    logits.copy_(randn(T + rule["E"], T, rule["E"], scale=1.5))       # in 16 bits equal logits are frequent
    check_route(ctx, logits, rule)


@pytest.mark.parametrize("rule", RULES)
def test_router_masks(ctx, rule):
    """Rows with nothing left, with one expert, fewer than k, NaN, +infinity, the lowest number, all equal, +-0."""
    E = rule["E"]
    x = randn(E, 12, E)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, E // 2] = 0.3
    x[2, ::2] = -math.inf
    x[3, ::3] = math.nan
    x[4] = math.nan
    x[5, E - 1] = math.inf
    x[6] = torch.finfo(F32).min
    x[7] = 0.25
    x[8, ::2], x[8, 1::2] = 0.0, -0.0
    x[9] = -math.inf
    x[9, : (E + 3) // 4] = -1.0
    x[10, : E // 2] = torch.finfo(F32).min
    check_route(ctx, x, rule)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_best", [1, 2])
def test_router_near_ties(ctx, score, group_best):
    """Keys that 32 bits cannot tell apart: logits one step apart, biases that nearly cancel differences of scores, and
    pairs of experts that are equal in everything."""
    E, T = 64, 200
    x = randn(1, T, E, scale=0.5)
    x[:, 1::2] = torch.nextafter(x[:, ::2], torch.full_like(x[:, ::2], math.inf))
    x[::3, 1::2] = x[::3, ::2]
    bias = randn(2, E, scale=0.05)
    bias[1::2] = bias[::2]
    # rows whose scores differ between two experts by what the bias gives back, up to a part in 2^24 and more
    far = plain.f64(x)
    p = 1 / (1 + np.exp(-far[7])) if score == "sigmoid" else np.exp(far[7] - far[7].max()) / np.exp(far[7] - far[7].max()).sum()
    bias[5], bias[9] = float(0.3 - p[5]), float(0.3 - p[9])
    for b in (None, bias):
        args = dict(score=score, n_groups=8, top_groups=3, group_best=group_best, renormalize=True, scale=1.0)
        ids, gates = ctx.pw_route_tokens(x, 6, bias=b, **args)
        ref_ids, ref_gates = plain.route(x, 6, bias=None if b is None else plain.f64(b), **args)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        np.testing.assert_allclose(gates.cpu().numpy(), ref_gates, rtol=52 * U)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_best", [1, 2])
@pytest.mark.parametrize("E,n_groups,top_groups", [(256, 8, 4), (160, 8, 3), (96, 3, 2), (64, 32, 7), (256, 16, 15), (250, 2, 1), (128, 64, 5)])
def test_router_groups_close(ctx, score, group_best, E, n_groups, top_groups):
    """Groups whose scores differ by a few steps of 32 bits or not at all: the same logits in every group, in another
    order, some of them moved by up to three steps; in a third of the rows one group is far above, one masked."""
    T, per = 120, E // n_groups
    gen = torch.Generator().manual_seed(E + n_groups)
    base = torch.randn(T, 1, per, generator=gen).expand(T, n_groups, per).clone()
    for _ in range(3):
        move = torch.rand(base.shape, generator=gen) < 0.3
        base = torch.where(move, torch.nextafter(base, torch.full_like(base, math.inf)), base)
    base[1::3, n_groups // 2] += 0.5
    base[2::3, n_groups - 1] = -math.inf
    bias = torch.randn(per, generator=gen) * 0.1               # goes with the logit
    order = torch.argsort(torch.rand(n_groups, per, generator=gen), dim=1)
    x = torch.gather(base, 2, order.expand(T, n_groups, per)).reshape(T, E).cuda()
    for b in (None, bias[order].reshape(E).cuda()):
        args = dict(score=score, n_groups=n_groups, top_groups=top_groups, group_best=group_best, renormalize=True, scale=1.0)
        k = min(8, top_groups * per)
        ids, gates = ctx.pw_route_tokens(x, k, bias=b, **args)
        ref_ids, ref_gates = plain.route(x, k, bias=None if b is None else plain.f64(b), **args)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        np.testing.assert_allclose(gates.cpu().numpy(), ref_gates, rtol=52 * U)


def test_router_agrees_with_the_layers_own_rule(ctx):
    cfg = synth.CONFIGS["finegrained_decode"]
    logits = synth.router_logits(cfg, device="cuda")
    ids, gates = ctx.pw_route_tokens(logits, cfg.top_k)
    own = B.pw_route_tokens_static(logits, cfg.top_k)
    assert torch.equal(ids, own["topk_ids"])
    np.testing.assert_allclose(gates.cpu().numpy(), own["gates"].cpu().numpy(), rtol=1e-6, atol=1e-9)


# ---- layer call with a given routing ---------------------------------------------------------------

SMALL = synth.LayerConfig("ops_small", 16, 4, 256, 384, 200, n_shared=2, routing="zipf", zipf_a=1.2, bit_rule="int4_10fp16_20int2")


@pytest.mark.parametrize("mode", [B.PW_MODE_SIMT, B.PW_MODE_TENSOR])
@pytest.mark.parametrize("T", [1, 5, 200])
def test_routed_layer_gives_the_bits_of_the_layer(mode, T):
    c = make_ctx(SMALL, max_tokens=T)
    try:
        pages, _ = build_layer(c, SMALL)
        x, logits = synth.activations(SMALL, device="cuda", tokens=T), synth.router_logits(SMALL, device="cuda", tokens=T)
        want = c.pw_moe_forward(0, x, logits, SMALL.top_k, mode=mode)
        r = c.pw_get_routing(T, SMALL.top_k)
        got = c.pw_moe_forward_routed(0, x, r["topk_ids"], r["gates"], mode=mode)
        assert torch.equal(got, want)
        again = c.pw_get_routing(T, SMALL.top_k)
        assert all(torch.equal(r[n], again[n]) for n in r)
        assert c.pw_last_device_status() == 0
    finally:
        c.close()


def near(got, want):
    """The tolerance of the layer: the two calls give an expert other numbers of tokens, so its sums other orders."""
    max_abs, rel = error_metrics(got.cpu().numpy(), want.cpu().numpy())
    assert max_abs <= 2e-2 and rel <= 5e-3, (max_abs, rel)


@pytest.mark.parametrize("mode", [B.PW_MODE_SIMT, B.PW_MODE_TENSOR])
@pytest.mark.parametrize("T,n_shared", [(1, 0), (1, 2), (37, 2), (200, 2), (200, 0)])
def test_routed_layer_skips_pairs_without_an_expert(mode, T, n_shared):
    cfg = synth.LayerConfig("ops_skip", 16, 4, 256, 384, T, n_shared=n_shared, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x = synth.activations(cfg, device="cuda")
        ids, gates = c.pw_route_tokens(synth.router_logits(cfg, device="cuda"), 4)
        drop = torch.rand(T, 4, generator=gen(T), device="cuda") < 0.4
        drop[0] = True                                                 # a token without any expert
        kept = torch.where(drop, torch.zeros_like(gates), gates)
        want = c.pw_moe_forward_routed(0, x, ids, kept, mode=mode)     # the same experts with gate 0
        holes = torch.where(drop, torch.full_like(ids, -1), ids)
        loud = torch.where(drop, torch.full_like(gates, math.nan), gates)   # the gate of a hole is not looked at
        acc = c.pw_observe(True)
        got = c.pw_moe_forward_routed(0, x, holes, loud, mode=mode)
        near(got, want)
        r = {n: v.cpu().numpy() for n, v in c.pw_get_routing(T, 4).items()}
        h = holes.cpu().numpy()
        counts = np.bincount(h[h >= 0], minlength=16)
        assert np.array_equal(r["counts"], counts) and np.array_equal(r["offsets"], np.concatenate([[0], np.cumsum(counts)]))
        order = [p for e in range(16) for p in np.flatnonzero(h.reshape(-1) == e)]
        assert np.array_equal(r["perm"], np.array(order + [-1] * (T * 4 - len(order))))
        pairs = acc[0, :, B.OBS_FIELD_NAMES.index("pairs")].cpu().numpy()
        assert np.array_equal(pairs, np.concatenate([counts, np.full(n_shared, T)]))
        assert c.pw_last_device_status() == 0
        # an id that is no expert is reported and skipped
        holes[drop] = 16
        holes[0, 0] = -7
        assert torch.equal(c.pw_moe_forward_routed(0, x, holes, gates, mode=mode), got)
        assert c.pw_last_device_status() == 1
        # the same expert twice
        twice = ids.clone()
        twice[:, 1] = twice[:, 0]
        once = gates.clone()
        once[:, 0] += once[:, 1]
        once[:, 1] = 0
        a, b = c.pw_moe_forward_routed(0, x, twice, gates, mode=mode), c.pw_moe_forward_routed(0, x, twice, once, mode=mode)
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-4)
    finally:
        c.close()


@pytest.mark.parametrize("mode", [B.PW_MODE_SIMT, B.PW_MODE_TENSOR])
@pytest.mark.parametrize("T", [1, 9, 200])
def test_routed_layer_with_an_expert_twice(mode, T):
    """A caller's routing may name an expert twice, and one expert in every pair: its gates add up."""
    cfg = synth.LayerConfig("ops_twice", 16, 4, 256, 384, T, n_shared=1, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x = synth.activations(cfg, device="cuda")
        ids, gates = c.pw_route_tokens(synth.router_logits(cfg, device="cuda"), 4)
        for same in ([0, 0, 2, 3], [0, 0, 0, 0]):
            twice = ids[:, same] if same[2] else torch.full_like(ids, 11)
            once, sums = twice.clone(), gates.clone()
            for j in range(3, 0, -1):
                dup = twice[:, j] == twice[:, 0]
                once[dup, j] = -1
                sums[:, 0] += torch.where(dup, gates[:, j], torch.zeros_like(gates[:, j]))
            near(c.pw_moe_forward_routed(0, x, twice, gates, mode=mode), c.pw_moe_forward_routed(0, x, once, sums, mode=mode))
        assert c.pw_last_device_status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("mode", [B.PW_MODE_SIMT, B.PW_MODE_TENSOR])
def test_routed_layer_replayed_with_other_ids(mode):
    """Router and experts captured together: a replay takes the logits that are there then."""
    cfg = synth.LayerConfig("ops_graph", 16, 4, 256, 384, 33, n_shared=1, bit_rule="int4_10fp16_20int2")
    c = make_ctx(cfg)
    try:
        pages, _ = build_layer(c, cfg)
        x, out = synth.activations(cfg, device="cuda"), torch.empty(33, 256, device="cuda")
        ids, gates = torch.empty(33, 4, dtype=torch.int32, device="cuda"), torch.empty(33, 4, device="cuda")
        logits = torch.zeros(33, 16, device="cuda")
        s = torch.cuda.Stream()
        step = lambda: (c.pw_route_tokens(logits, 4, ids=ids, gates=gates, stream=s), c.pw_moe_forward_routed(0, x, ids, gates, out=out, mode=mode, stream=s))
        with torch.cuda.stream(s):
            step()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
        for seed in (3, 4):
            logits.copy_(randn(seed, 33, 16))
            logits[7] = -math.inf                                      # a token without any expert
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            got, i, w = out.clone(), ids.clone(), gates.clone()
            assert bool((i[7] == -1).all())
            assert torch.equal(c.pw_moe_forward_routed(0, x, i, w, mode=mode), got)
        assert c.pw_last_device_status() == 0
    finally:
        c.close()


def test_routed_layer_refuses(ctx):
    x = torch.zeros(4, 256, dtype=F16, device="cuda")
    ids, gates = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for bad in ((x[:, :128].contiguous(), ids, gates), (x, ids.long(), gates), (x, ids, gates.half()), (x, ids[:3], gates), (x, ids, gates[:, :1]),
                (x, ids.cpu(), gates), (x.t().contiguous().t(), ids, gates)):
        with pytest.raises(B.PwError):
            ctx.pw_moe_forward_routed(0, *bad)
    with pytest.raises(B.PwError) as e:                                # nothing published
        ctx.pw_moe_forward_routed(0, x, ids, gates)
    assert e.value.status == 5


# ---- together --------------------------------------------------------------------------------------

def test_one_layer_from_stream_to_stream(orc):
    """Residual stream -> norm -> 8-bit router product -> routing -> layer -> residual stream and next norm, each step
    against its definition on what the step before it produced."""
    cfg = SMALL
    T = 50
    c = make_ctx(cfg, max_tokens=T)
    try:
        pages, _ = build_layer(c, cfg)
        wr, swr = c.pw_quantize_scaled(randn(1, cfg.n_experts, cfg.hidden, scale=0.05, dtype=F16), 128)
        stream = randn(2, T, cfg.hidden, dtype=F16)
        attn = randn(3, T, cfg.hidden, scale=0.3)
        w = (1 + randn(4, cfg.hidden, scale=0.1)).to(F16)
        bias = randn(5, cfg.n_experts, scale=0.1)
        hidden, after = torch.empty_like(stream), torch.empty_like(stream)
        q, qs = B.scaled_empty(T, cfg.hidden, 1)
        rule = dict(score="sigmoid", n_groups=4, top_groups=2, group_best=2, renormalize=True, scale=2.5)

        def step(s=None):
            c.pw_add_rmsnorm(attn, w, 1e-6, residual=stream, residual_out=after, y=hidden, q=q, q_scales=qs, stream=s)
            logits = c.pw_scaled_linear(q, qs, wr, swr, out_dtype=F32, stream=s)
            ids, gates = c.pw_route_tokens(logits, cfg.top_k, bias=bias, stream=s, **rule)
            out = c.pw_moe_forward_routed(0, hidden, ids, gates, stream=s)
            last = torch.empty_like(after)
            nxt = c.pw_add_rmsnorm(out, w, 1e-6, residual=after, residual_out=last, stream=s)[1]
            return logits, ids, gates, out, last, nxt

        logits, ids, gates, out, last, nxt = step()
        check_norm(attn, stream, w, 1e-6, after, hidden, q, qs)
        ref, mags = plain.linear(q, qs, wr, swr)
        assert np.all(np.abs(plain.f64(logits) - ref) <= mags * (4 * 2.0 ** -22 + (2 + 2 + 7) * U) + np.abs(ref) * U)
        ref_ids, ref_gates = plain.route(logits, cfg.top_k, bias=plain.f64(bias), **rule)
        assert np.array_equal(ids.cpu().numpy(), ref_ids)
        np.testing.assert_allclose(gates.cpu().numpy(), ref_gates, rtol=52 * U)
        # the oracle's layer takes logits; logits that are log gates on the chosen experts give these gates / their sum
        fake = np.full((T, cfg.n_experts), -1e4, np.float32)
        np.put_along_axis(fake, ref_ids, np.log(ref_gates / ref_gates.sum(1, keepdims=True)).astype(np.float32), 1)
        opages = [export_to_oracle(c, p, orc) for p in pages]
        hid = hidden.cpu().numpy()
        routed = orc.moe_forward(hid, fake, cfg.top_k, opages, n_shared=cfg.n_shared)
        shared_only = routed - orc.moe_forward(hid, fake, cfg.top_k, opages[: 3 * cfg.n_experts], n_shared=0)
        want = shared_only + 2.5 * (routed - shared_only)
        max_abs, rel = error_metrics(out.cpu().numpy(), want)
        assert max_abs <= 2.5 * 2e-2 and rel <= 5e-3, (max_abs, rel)    # the layer's tolerance, gates up to 2.5 times larger
        check_norm(out, after, w, 1e-6, last, nxt, None, None)

        # captured and replayed on another stream: the same bits, for new contents of the input buffers too
        want = [t.clone() for t in (logits, ids, gates, out, last, nxt)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
        keep = attn.clone()
        for t in got:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, v) for g, v in zip(got, want))
        attn.copy_(randn(9, T, cfg.hidden))
        graph.replay()
        torch.cuda.synchronize()
        new = [t.clone() for t in got]
        fresh = step()
        assert all(torch.equal(g, v) for g, v in zip(new, fresh)) and not torch.equal(new[3], want[3])
        attn.copy_(keep)
        with torch.cuda.stream(side):
            out2 = step(side)
        side.synchronize()
        assert all(torch.equal(g, v) for g, v in zip(out2, want))
        assert c.pw_last_device_status() == 0
        del graph
    finally:
        c.close()


def test_two_streams_at_once(ctx):
    jobs = []
    for i, (T, N, K) in enumerate(((64, 2048, 2048), (300, 1408, 2048))):
        a, sa, w, sw = operands(ctx, T, N, K, seed=10 * i)
        x, wt = randn(i, T, K), randn(i + 5, K)
        logits = randn(i + 9, T, 64)
        jobs.append((a, sa, w, sw, x, wt, logits))

    def work(j):
        a, sa, w, sw, x, wt, logits = j
        return ctx.pw_scaled_linear(a, sa, w, sw), ctx.pw_add_rmsnorm(x, wt)[1], *ctx.pw_route_tokens(logits, 6), *ctx.pw_quantize_scaled(x, 128)

    want = [work(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(20):
        for n, (s, j) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[n].append(work(j))
    torch.cuda.synchronize()
    for n in range(2):
        for r in got[n]:
            for g, v in zip(r, want[n]):
                assert torch.equal(g.view(torch.uint8) if g.element_size() == 1 else g, v.view(torch.uint8) if v.element_size() == 1 else v)


def test_no_rows(ctx):
    e = torch.empty
    q, s = ctx.pw_quantize_scaled(e(0, 300, device="cuda"), 1)
    assert q.shape == (0, 300) and s.shape == (0, 3)
    ctx.pw_add_rmsnorm(e(0, 300, device="cuda"), torch.ones(300, device="cuda"))
    w, sw = ctx.pw_quantize_scaled(randn(1, 40, 300), 128)
    assert ctx.pw_scaled_linear(q, s, w, sw).shape == (0, 40)
    assert ctx.pw_route_tokens(e(0, 8, device="cuda"), 2)[0].shape == (0, 2)
    torch.cuda.synchronize()


def test_binding_refuses(ctx):
    x = torch.zeros(4, 256, device="cuda")
    q, s = ctx.pw_quantize_scaled(x, 1)
    w, sw = ctx.pw_quantize_scaled(x, 128)
    for call in (lambda: ctx.pw_quantize_scaled(x.double(), 1), lambda: ctx.pw_quantize_scaled(x.cpu(), 1), lambda: ctx.pw_quantize_scaled(x, 64),
                 lambda: ctx.pw_quantize_scaled(x[0], 1), lambda: ctx.pw_quantize_scaled(x.t(), 1), lambda: ctx.pw_quantize_scaled(x[:, 1:], 1),
                 lambda: ctx.pw_quantize_scaled(x[:1].expand(4, 256), 1),
                 lambda: ctx.pw_quantize_scaled(x, 1, q=q), lambda: ctx.pw_quantize_scaled(x, 1, q=q, scales=sw),
                 lambda: ctx.pw_add_rmsnorm(x, x[0, :255]), lambda: ctx.pw_add_rmsnorm(x, x[0], residual=x[:3]),
                 lambda: ctx.pw_add_rmsnorm(x, x[0], residual=x, residual_out=x.half()), lambda: ctx.pw_add_rmsnorm(x, x[0], q=q),
                 lambda: ctx.pw_add_rmsnorm(x, x[0], residual_out=x), lambda: ctx.pw_add_rmsnorm(x, x[0], y=x[:, :128]),
                 lambda: ctx.pw_scaled_linear(q, sw, w, sw), lambda: ctx.pw_scaled_linear(q, s, w, s), lambda: ctx.pw_scaled_linear(q[:, :128], s, w, sw),
                 lambda: ctx.pw_scaled_linear(q, s, w, sw, out_dtype=torch.float64), lambda: ctx.pw_scaled_linear(x, s, w, sw),
                 lambda: ctx.pw_scaled_linear(q, s, w, sw, out=x), lambda: ctx.pw_route_tokens(x, 2, score="tanh"), lambda: ctx.pw_route_tokens(x, 0),
                 lambda: ctx.pw_route_tokens(x, 2, bias=x[0, :8]), lambda: ctx.pw_route_tokens(x, 2, ids=torch.zeros(4, 2, device="cuda")),
                 lambda: ctx.pw_route_tokens(x, 2, n_groups=3, top_groups=1), lambda: ctx.pw_route_tokens(x, 2, scale=math.inf)):
        with pytest.raises(B.PwError):
            call()
