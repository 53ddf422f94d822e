"""The products on weight pages and the layer in 64 bits (numpy), from what a page holds in the canonical layout, with bounds of
the errors that the calls for few tokens may make."""
import numpy as np
import torch

from paper_2607_16184_b200 import binding as B
from plain_operators import HALF_STEP, TINY_STEP, f64

GROUP = 128
# a name of a format -> bits, bit-planes
FORMATS = {"16": (16, False), "8": (8, False), "4": (4, False), "3": (3, False), "2": (2, False),
           "p4": (4, True), "p3": (3, True), "p2": (2, True)}


def make_page(ctx, w, fmt):
    bits, planes = FORMATS[fmt]
    return ctx.pw_quantize_planes(w).at(bits) if planes else ctx.pw_quantize_block(w, bits)


def stored(ctx, page):
    """(codes, scales, zero-points) per weight in 64 bits, out of the exported page; 16 bits: (weights, 1, 0)."""
    ex = ctx.pw_export_planes(page) if page.layout == B.PW_LAYOUT_PLANES else ctx.pw_export_page(page)
    torch.cuda.synchronize()
    raw = ex.codes.cpu().numpy()
    if page.bits == 16:
        w = raw.view(np.float16).reshape(page.rows, page.cols).astype(np.float64)
        return w, np.ones_like(w), np.zeros_like(w)
    stream = np.unpackbits(raw, bitorder="little").reshape(page.rows * page.cols, page.bits)
    codes = (stream.astype(np.int64) << np.arange(page.bits)).sum(1).reshape(page.rows, page.cols).astype(np.float64)
    wide = [np.repeat(f64(t).reshape(page.rows, -1), GROUP, 1) for t in (ex.scales, ex.zps)]
    return codes, wide[0], wide[1]


def weights(ctx, page):
    c, s, z = stored(ctx, page)
    return c * s + z


def product(x, block):
    """(x . w^T, bound of its error in fp32) for x [T, K] in 64 bits and a block from stored().

    A product code * x is exact.  On the way to the result it passes, besides the additions inside the tensor core, which
    cut at most the last bit of the larger operand (two half steps each): one accumulation per 16 columns, two or three
    joins, the scale, the groups' sum, the warps' and the CTAs' sums; sum x passes as many.  K / 8 + 64 half steps of the sum
    of magnitudes cover all of them."""
    c, s, z = (m[:, :x.shape[1]] for m in block)
    out = x @ (c * s + z).T
    size = np.abs(x) @ (np.abs(c * s) + np.abs(z)).T
    return out, size * (x.shape[1] / 8 + 64) * 2.0 ** -24


def rounded(values, bound, dtype):
    """The bound with the one rounding to the output's type."""
    return bound + np.maximum((np.abs(values) + bound) * HALF_STEP[dtype], TINY_STEP[dtype] / 2)


def layer(x, blocks, pairs, parts=1):
    """(out, bound) of the layer: x [T, H] in 64 bits, blocks[e] = three of stored(), pairs = (token, expert, gate).
    parts: fp16 numbers that h is rounded to; the second takes what the first leaves (at most 2^-11 of h) and is off by half
    a step of that."""
    out, bound = np.zeros_like(x), np.zeros_like(x)
    cache = {}
    for t, e, gate in pairs:
        if (t, e) not in cache:
            g, dg = product(x[t:t + 1], blocks[e][0])
            u, du = product(x[t:t + 1], blocks[e][1])
            with np.errstate(over="ignore"):
                silu = g / (1.0 + np.exp(-g))
            h = silu * u
            # the slope of silu is at most 1.1; its fast exponential and division: a few units of 2^-21, and all that may
            # be lost where exp(-g) overflows is less than 2^-24
            dh = (1.1 * dg + np.abs(silu) * 2.0 ** -19 + 2.0 ** -24) * (np.abs(u) + du) + np.abs(silu) * du
            dh = dh + np.maximum((np.abs(h) + dh) * HALF_STEP[torch.float16] ** parts, TINY_STEP[torch.float16] / 2)
            y, dy = product(h, blocks[e][2])
            c, s, z = blocks[e][2]
            cache[t, e] = y[0], dy[0] + (dh @ np.abs(c * s + z).T)[0] * 1.001
        y, dy = cache[t, e]
        out[t] += gate * y
        bound[t] += abs(gate) * (dy + np.abs(y) * 2.0 ** -20)   # gates: fp32, from an exponential and a division
    return out, bound


def routing(logits, k):
    """The layer call's own rule: (token, expert, gate)."""
    pairs = []
    for t, row in enumerate(logits):
        row = np.where(np.isnan(row), -np.inf, row)
        best = sorted(range(len(row)), key=lambda e: (-row[e], e))[:k]
        p = np.exp(row[best] - row[best[0]])
        pairs += [(t, e, g) for e, g in zip(best, p / p.sum())]
    return pairs
