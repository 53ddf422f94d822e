"""The operators around the layer in 64 bits (numpy), written from their definitions: what the GPU tests compare with."""
import math

import numpy as np
import torch

GROUP = 128
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY_STEP = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}   # spacing of subnormals


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def rounding(values, dtype):
    """Largest error of one rounding of these values to a type: half a step, or half of the subnormal spacing."""
    return np.maximum(np.abs(values) * HALF_STEP[dtype], TINY_STEP[dtype] / 2)


def rmsnorm(x, residual, w, eps):
    s = f64(x) + (0.0 if residual is None else f64(residual))
    return s, s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * f64(w)[None, :]


def block_tops(y, block_rows):
    """Largest magnitude of every block, [row blocks, column blocks]."""
    R, C = y.shape
    out = np.zeros((-(-R // block_rows), -(-C // GROUP)))
    for i in range(out.shape[0]):
        for g in range(out.shape[1]):
            out[i, g] = np.abs(y[i * block_rows:(i + 1) * block_rows, g * GROUP:(g + 1) * GROUP]).max()
    return out


def spread(scales, block_rows, shape):
    """Scales per element."""
    return np.repeat(np.repeat(scales, block_rows, 0), GROUP, 1)[:shape[0], :shape[1]]


def quantize_bits(x, block_rows):
    """(codes as uint8, scales fp32) exactly as defined: fp32 operations, one rounding each."""
    v = x.detach().float().cpu().numpy()
    tops = block_tops(v, block_rows).astype(np.float32)
    scales = np.maximum(tops / np.float32(448), np.float32(2.0 ** -126)).astype(np.float32)
    scales[tops == 0] = 1
    r = (np.float32(1) / scales).astype(np.float32)
    q = torch.from_numpy((v * spread(r, block_rows, v.shape)).astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).numpy(), scales


def code_values(q):
    return q.contiguous().view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)


def linear(a, a_scales, w, w_scales):
    """(out, sum of magnitudes) in 64 bits."""
    A = code_values(a) * spread(f64(a_scales), 1, a.shape)
    W = code_values(w) * spread(f64(w_scales), GROUP, w.shape)
    return A @ W.T, np.abs(A) @ np.abs(W).T


def route(logits, top_k, score, bias, n_groups, top_groups, group_best, renormalize, scale):
    x = np.minimum(f64(logits), np.finfo(np.float32).max)
    T, E = x.shape
    per = E // n_groups
    ids, gates = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    for t in range(T):
        open_ = [e for e in range(E) if x[t, e] > -np.inf]
        if score == "softmax":
            m = max([x[t, e] for e in open_], default=0.0)
            p = {e: math.exp(x[t, e] - m) for e in open_}
            total = sum(p.values())
            p = {e: v / total for e, v in p.items()}
        else:
            p = {e: 1.0 / (1.0 + math.exp(-x[t, e])) if x[t, e] > -700 else 0.0 for e in open_}
        sums = {e: p[e] + (0.0 if bias is None else float(bias[e])) for e in open_}
        key = {e: x[t, e] for e in open_} if bias is None else sums     # without a bias: the order of the logits
        if n_groups > 1:
            best = {}
            for e in open_:
                best.setdefault(e // per, []).append(key[e] if group_best == 1 else sums[e])
            rank = sorted(best, key=lambda g: (-sum(sorted(best[g], reverse=True)[:group_best]), g))[:top_groups]
            open_ = [e for e in open_ if e // per in rank]
        chosen = sorted(open_, key=lambda e: (-key[e], e))[:top_k]
        total = sum(p[e] for e in chosen) if renormalize else 1.0
        if renormalize and score == "softmax" and chosen:   # the same ratio, where the scores themselves underflow
            m = max(x[t, e] for e in chosen)
            p = {e: math.exp(x[t, e] - m) for e in chosen}
            total = sum(p.values())
        for j, e in enumerate(chosen):
            ids[t, j], gates[t, j] = e, (p[e] / total if total > 0 else 0.0) * scale
    return ids, gates
