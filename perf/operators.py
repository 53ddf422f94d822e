"""The operators around a paged-weight MoE layer, as they are measured: the residual's addition with the root-mean-square
norm (and an 8-bit output with scales), the quantizer of the scaled 8-bit format, the router with scores, bias and groups,
and the matrix product of two scaled 8-bit matrices.

A scaled 8-bit matrix is e4m3 codes with an fp32 scale per block of 128 columns and one row (activations) or 128 rows
(weights); the last block of an odd size is short.  ``run`` computes the plain form of an operator, or, where ``own`` is
true, calls the library.
"""
import math

import numpy as np
import torch

own = False

GROUP = 128
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
TINY = 2.0 ** -126


def listed():
    return [
        # one token of a decode step behind an 8-expert layer of width 4096
        {"name": "norm_one_token", "op": "norm", "tokens": 1, "hidden": 4096, "x": "f32", "res": "f16", "y": "f16", "quant": False},
        # a decode batch of the fine-grained layer, a width that is no multiple of the group, both outputs
        {"name": "norm_batch_odd", "op": "norm", "tokens": 257, "hidden": 2056, "x": "f32", "res": "bf16", "y": "f16", "quant": True},
        # a prompt of 4096 tokens: norm for the experts' input and the 8-bit copy for the dense products
        {"name": "norm_prompt", "op": "norm", "tokens": 4096, "hidden": 4096, "x": "f32", "res": "f16", "y": "f16", "quant": True},
        # activations of a decode batch, quantized on their way into a dense product
        {"name": "quantize_activations", "op": "quantize", "rows": 256, "cols": 1408, "x": "f16", "block_rows": 1},
        # a weight matrix quantized when a model is loaded
        {"name": "quantize_weights", "op": "quantize", "rows": 14336, "cols": 4096, "x": "f16", "block_rows": 128},
        # one token over 8 experts, the softmax router of the 8-expert layer
        {"name": "route_one_token", "op": "route", "tokens": 1, "experts": 8, "top_k": 2, "logits": "f32", "score": "softmax",
         "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "renormalize": True, "scale": 1.0, "padding": 0},
        # a padded decode batch of the fine-grained layer: the rows of the padding have every expert masked
        {"name": "route_padded_batch", "op": "route", "tokens": 256, "experts": 64, "top_k": 6, "logits": "bf16", "score": "softmax",
         "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "renormalize": False, "scale": 1.0, "padding": 19},
        # a prompt through a sigmoid router with a balancing bias and groups of experts
        {"name": "route_prompt_groups", "op": "route", "tokens": 4096, "experts": 256, "top_k": 8, "logits": "f32", "score": "sigmoid",
         "bias": True, "groups": 8, "top_groups": 4, "group_best": 2, "renormalize": True, "scale": 2.5, "padding": 0},
        # a dense projection for one token
        {"name": "linear_one_token", "op": "linear", "tokens": 1, "out_features": 4096, "in_features": 4096, "out": "f16"},
        # the widest projection for a decode batch of 64: the weights' bytes count
        {"name": "linear_decode", "op": "linear", "tokens": 64, "out_features": 14336, "in_features": 4096, "out": "f16"},
        # router logits of an odd batch: few columns, fp32 out, a contraction with a short last block
        {"name": "linear_router_odd", "op": "linear", "tokens": 301, "out_features": 64, "in_features": 2056, "out": "f32"},
        # a prompt of 4096 tokens through the widest projection
        {"name": "linear_prompt", "op": "linear", "tokens": 4096, "out_features": 14336, "in_features": 4096, "out": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "quantize", "route", "linear", "linear"))
    if op == "norm":
        hidden = _log_int(rng, 100, 14336)
        if rng.random() < 0.5:
            hidden = max(128, hidden // 128 * 128)
        tokens = _log_int(rng, 1, max(1, min(4096, 4096 * 4096 // hidden)))
        quant = rng.random() < 0.5
        return {"op": op, "tokens": tokens, "hidden": hidden, "x": rng.choice(("f32", "f16", "bf16")),
                "res": rng.choice(("f32", "f16", "bf16", "none")), "y": rng.choice(("f16", "bf16", "none") if quant else ("f16", "bf16", "f32")),
                "quant": quant}
    if op == "quantize":
        cols = _log_int(rng, 100, 14336)
        return {"op": op, "rows": _log_int(rng, 1, min(14336, 14336 * 4096 // cols)), "cols": cols,
                "x": rng.choice(("f32", "f16", "bf16")), "block_rows": rng.choice((1, 128))}
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        per = _log_int(rng, max(2, 8 // groups), 256 // groups)
        top_groups = rng.randint(1, groups)
        return {"op": op, "tokens": _log_int(rng, 1, 4096), "experts": groups * per, "top_k": rng.randint(1, min(8, top_groups * per)),
                "logits": rng.choice(("f32", "f16", "bf16")), "score": rng.choice(("softmax", "sigmoid")), "bias": rng.random() < 0.5,
                "groups": groups, "top_groups": top_groups, "group_best": rng.choice((1, 2)), "renormalize": rng.random() < 0.5,
                "scale": rng.choice((1.0, 2.5)), "padding": 0}
    n, k = _log_int(rng, 8, 14336), _log_int(rng, 64, 14336)
    k = min(k, 14336 * 4096 // n)
    if rng.random() < 0.5:
        n, k = max(8, n // 8 * 8), max(128, k // 128 * 128)
    return {"op": op, "tokens": _log_int(rng, 1, 4096), "out_features": n, "in_features": k, "out": rng.choice(("f16", "bf16", "f32"))}


# ---- the scaled 8-bit format in plain torch --------------------------------------------------------

def _padded(n, to):
    return -(-n // to) * to


def _codes_buffer(rows, cols, device):
    """e4m3 [rows, cols] whose rows start 16 bytes apart or a multiple of that, as the product's operands have them."""
    return torch.zeros(rows, _padded(cols, 16), dtype=torch.uint8, device=device).view(E4M3)[:, :cols]


def _quantize(x, block_rows):
    """(codes e4m3 [rows, cols], scales f32 [row blocks, column blocks]) of a matrix in 32 bits."""
    rows, cols = x.shape
    R, G = _padded(rows, block_rows), _padded(cols, GROUP)
    p = torch.nn.functional.pad(x, (0, G - cols, 0, R - rows)).reshape(R // block_rows, block_rows, G // GROUP, GROUP)
    top = p.abs().amax(dim=(1, 3), keepdim=True)
    scale = torch.where(top == 0, torch.ones_like(top), (top / E4M3_MAX).clamp_min(TINY))
    q = (p / scale).reshape(R, G)[:rows, :cols]
    return q.to(E4M3), scale.reshape(R // block_rows, G // GROUP)


def _values(q, scales, block_rows):
    """What the codes stand for, in 32 bits."""
    rows, cols = q.shape
    s = scales.repeat_interleave(GROUP, 1)[:, :cols]
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, 0)[:rows]
    return q.float() * s


# ---- inputs ----------------------------------------------------------------------------------------

def prepare(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=d)

    s = dict(case)
    op = case["op"]
    if op == "norm":
        T, H = case["tokens"], case["hidden"]
        # the layer's output is small next to the residual stream, which has a few large channels
        s["x_t"] = (normal(T, H) * 0.5).to(TYPES[case["x"]])
        loud = 1.0 + 20.0 * (torch.rand(H, generator=g, device=d) < 0.005)
        s["res_t"] = (normal(T, H) * loud).to(TYPES[case["res"]]) if case["res"] != "none" else None
        s["w_t"] = (1.0 + 0.2 * normal(H)).to(TYPES["f32" if case["res"] in ("f32", "none") else case["res"]])
        s["eps"] = 1e-6
        s["res_out"] = torch.empty_like(s["res_t"]) if s["res_t"] is not None else None
        s["y_out"] = torch.empty(T, H, dtype=TYPES[case["y"]], device=d) if case["y"] != "none" else None
        s["q_out"] = _codes_buffer(T, H, d) if case["quant"] else None
        s["q_scales"] = torch.empty(T, _padded(H, GROUP) // GROUP, device=d) if case["quant"] else None
    elif op == "quantize":
        R, K = case["rows"], case["cols"]
        x = normal(R, K)
        if case["block_rows"] > 1:                       # weights: small, one in a thousand ten times larger
            x = x * 0.02 * (1.0 + 9.0 * (torch.rand(R, K, generator=g, device=d) < 0.001))
        s["x_t"] = x.to(TYPES[case["x"]])
        s["q_out"] = _codes_buffer(R, K, d)
        s["q_scales"] = torch.empty(_padded(R, case["block_rows"]) // case["block_rows"], _padded(K, GROUP) // GROUP, device=d)
    elif op == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        x = normal(T, E) * 1.5
        if case["padding"]:
            x[T - case["padding"]:] = -math.inf
        s["x_t"] = x.to(TYPES[case["logits"]])
        s["bias_t"] = normal(E) * 0.05 if case["bias"] else None
        s["ids"] = torch.empty(T, k, dtype=torch.int32, device=d)
        s["gates"] = torch.empty(T, k, device=d)
    else:
        T, N, K = case["tokens"], case["out_features"], case["in_features"]
        a, s["a_scales"] = _quantize(normal(T, K), 1)
        w, s["w_scales"] = _quantize(normal(N, K) * 0.02, GROUP)
        s["a"], s["w"] = _codes_buffer(T, K, d), _codes_buffer(N, K, d)
        s["a"].copy_(a)
        s["w"].copy_(w)
        s["out_t"] = torch.empty(T, N, dtype=TYPES[case["out"]], device=d)
    return s


# ---- one pass --------------------------------------------------------------------------------------

_context = None


def _library():
    """The context that a program keeps for as long as it runs (8 experts of 256 x 512: its workspace is small)."""
    global _context
    from paper_2607_16184_b200 import binding
    if _context is None:
        _context = binding.Context(1, 8, 0, 256, 512, 16, 2)
    return _context


def run(state):
    op = state["op"]
    if own:
        ctx = _context or _library()
        if op == "norm":
            ctx.pw_add_rmsnorm(state["x_t"], state["w_t"], state["eps"], residual=state["res_t"], residual_out=state["res_out"],
                               y=state["y_out"], q=state["q_out"], q_scales=state["q_scales"])
            return {"residual": state["res_out"], "y": state["y_out"], "q": state["q_out"], "q_scales": state["q_scales"]}
        if op == "quantize":
            ctx.pw_quantize_scaled(state["x_t"], state["block_rows"], q=state["q_out"], scales=state["q_scales"])
            return {"q": state["q_out"], "q_scales": state["q_scales"]}
        if op == "route":
            ctx.pw_route_tokens(state["x_t"], state["top_k"], score=state["score"], bias=state["bias_t"], n_groups=state["groups"],
                                top_groups=state["top_groups"], group_best=state["group_best"], renormalize=state["renormalize"],
                                scale=state["scale"], ids=state["ids"], gates=state["gates"])
            return {"ids": state["ids"], "gates": state["gates"]}
        ctx.pw_scaled_linear(state["a"], state["a_scales"], state["w"], state["w_scales"], out=state["out_t"])
        return {"out": state["out_t"]}
    return {"norm": _norm, "quantize": _quantize_case, "route": _route, "linear": _linear}[op](state)


def _norm(s):
    z = s["x_t"].float()
    out = {"residual": None, "y": None, "q": None, "q_scales": None}
    if s["res_t"] is not None:
        z = z + s["res_t"].float()
        out["residual"] = z.to(s["res_t"].dtype)
    y = z * torch.rsqrt(z.square().mean(1, keepdim=True) + s["eps"]) * s["w_t"].float()
    if s["y"] != "none":
        out["y"] = y.to(TYPES[s["y"]])
    if s["quant"]:
        out["q"], out["q_scales"] = _quantize(y, 1)
    return out


def _quantize_case(s):
    q, scales = _quantize(s["x_t"].float(), s["block_rows"])
    return {"q": q, "q_scales": scales}


def _route(s):
    # in 64 bits: which of two near scores is the larger one decides whole numbers
    x = s["x_t"].double()
    T, E = x.shape
    masked = torch.isnan(x) | (x == -math.inf)
    x = x.masked_fill(masked, -math.inf)
    if s["score"] == "softmax":
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        p = 1.0 / (1.0 + torch.exp(-x))
    key = p if s["bias_t"] is None else p + s["bias_t"].double()
    key = key.masked_fill(masked, -math.inf)
    if s["groups"] > 1:
        best = key.reshape(T, s["groups"], -1).sort(dim=2, descending=True).values[:, :, :s["group_best"]]
        none = best[:, :, 0] == -math.inf
        score = torch.where(best == -math.inf, torch.zeros_like(best), best).sum(2).masked_fill(none, -math.inf)
        kept = score.sort(dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        left = torch.zeros(T, s["groups"], dtype=torch.bool, device=x.device).scatter_(1, kept, True)
        key = key.masked_fill(~left.repeat_interleave(E // s["groups"], 1), -math.inf)
    order = key.sort(dim=1, descending=True, stable=True)
    ids, chosen = order.indices[:, :s["top_k"]], order.values[:, :s["top_k"]] > -math.inf
    gates = p.gather(1, ids).masked_fill(~chosen, 0.0)
    if s["renormalize"]:
        gates = gates / gates.sum(1, keepdim=True).clamp_min(1e-300)
    return {"ids": ids.masked_fill(~chosen, -1).int(), "gates": (gates * s["scale"]).float()}


def _linear(s):
    a, w = _values(s["a"], s["a_scales"], 1), _values(s["w"], s["w_scales"], GROUP)
    return {"out": (a @ w.t()).to(TYPES[s["out"]])}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2, "none": 0}
    op = case["op"]
    if op == "norm":
        T, H = case["tokens"], case["hidden"]
        w = size["f32" if case["res"] in ("f32", "none") else case["res"]]
        n = T * H * (size[case["x"]] + 2 * size[case["res"]] + size[case["y"]]) + w * H
        return {"bytes": n + (T * H + 4 * T * _padded(H, GROUP) // GROUP if case["quant"] else 0), "flops": 6 * T * H}
    if op == "quantize":
        R, K, b = case["rows"], case["cols"], case["block_rows"]
        return {"bytes": R * K * (size[case["x"]] + 1) + 4 * (_padded(R, b) // b) * (_padded(K, GROUP) // GROUP), "flops": 3 * R * K}
    if op == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": T * E * size[case["logits"]] + 8 * T * k + (4 * E if case["bias"] else 0), "flops": 10 * T * E}
    T, N, K = case["tokens"], case["out_features"], case["in_features"]
    G = _padded(K, GROUP) // GROUP
    return {"bytes": T * K + N * K + 4 * G * (T + _padded(N, GROUP) // GROUP) + size[case["out"]] * T * N, "flops": 2 * T * N * K}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_codes(y, block_rows):
    """Codes and scales of a matrix in 64 bits, block by block of columns."""
    rows, cols = y.shape
    q, scales = torch.empty(rows, cols, dtype=torch.float64, device=y.device), []
    for c in range(0, cols, GROUP):
        part = y[:, c:c + GROUP]
        top = part.abs().amax(1)
        top = torch.stack([t.max() for t in top.split(block_rows)]) if block_rows > 1 else top
        scale = (top / E4M3_MAX).clamp_min(TINY)
        scale[top == 0] = 1.0
        v = part / (scale.repeat_interleave(block_rows)[:rows, None])
        # nearest e4m3 value, ties to even: three mantissa bits down to exponent -6, a fixed step below it
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
        q[:, c:c + GROUP] = (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)
        scales.append(scale)
    return q, torch.stack(scales, 1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        z = s["x_t"].double()
        out = {"residual": None, "y": None, "q": None, "q_scales": None}
        if s["res_t"] is not None:
            z += s["res_t"].double()
            out["residual"] = z
        y = z / torch.sqrt((z * z).sum(1, keepdim=True) / case["hidden"] + s["eps"])
        y = y * s["w_t"].double()[None, :]
        if case["y"] != "none":
            out["y"] = y
        if case["quant"]:
            out["q"], out["q_scales"] = _exact_codes(y, 1)
        return out
    if op == "quantize":
        q, scales = _exact_codes(s["x_t"].double(), case["block_rows"])
        return {"q": q, "q_scales": scales}
    if op == "route":
        x = s["x_t"].double().cpu().numpy()
        bias = np.zeros(x.shape[1]) if s["bias_t"] is None else s["bias_t"].double().cpu().numpy()
        k, per = case["top_k"], x.shape[1] // case["groups"]
        ids, gates = np.full((len(x), k), -1, np.int32), np.zeros((len(x), k))
        for t, row in enumerate(x):
            open_ = [e for e in range(len(row)) if row[e] > -np.inf]
            if case["score"] == "softmax":
                e = np.exp(row - row[open_].max()) if open_ else row
                p = e / e[open_].sum() if open_ else e
            else:
                p = 1.0 / (1.0 + np.exp(-row))
            key = p + bias
            if case["groups"] > 1:
                by = {}
                for e in open_:
                    by.setdefault(e // per, []).append(key[e])
                rank = sorted(by, key=lambda j: (-sum(sorted(by[j])[::-1][:case["group_best"]]), j))[:case["top_groups"]]
                open_ = [e for e in open_ if e // per in rank]
            best = sorted(open_, key=lambda e: (-key[e], e))[:k]
            total = sum(p[e] for e in best) if case["renormalize"] else 1.0
            for j, e in enumerate(best):
                ids[t, j], gates[t, j] = e, p[e] / total * case["scale"]
        return {"ids": ids, "gates": gates}
    T, N, K = case["tokens"], case["out_features"], case["in_features"]
    out = torch.zeros(T, N, dtype=torch.float64, device="cuda")
    for g in range(_padded(K, GROUP) // GROUP):
        cut = slice(g * GROUP, min(K, (g + 1) * GROUP))
        w = s["w"][:, cut].double() * s["w_scales"][:, g].double().repeat_interleave(GROUP)[:N, None]
        out += s["a"][:, cut].double() * s["a_scales"][:, g].double()[:, None] @ w.t()
    return {"out": out}
