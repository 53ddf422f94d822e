"""Products on weight pages for few tokens, as they are measured: the dense product of a few tokens with the blocks of one or
several pages, and the whole mixture-of-experts layer for a few tokens.

A page holds a block [rows, cols] as a little-endian stream of codes with an fp16 scale and zero-point per row and group of
128 columns, weight = code * scale + zero-point (16 bits: the fp16 weights themselves); read from overlaid bit-planes the
code is the first bits of a 4-bit code.  Rows and columns of a page are multiples of 128; a block of other sizes is padded
with zeros.  ``run`` computes the plain form of an operator, or, where ``own`` is true, calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 128
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
# how a block is stored: codes of 16, 8, 4, 3 or 2 bits, or overlaid bit-planes read at 4, 3 or 2 bits
FORMATS = {"16": (16, False), "8": (8, False), "4": (4, False), "3": (3, False), "2": (2, False), "p4": (4, True), "p3": (3, True), "p2": (2, True)}
# the formats of a layer's routed blocks, dealt out in these shares
MIXES = {"mix": "16 16 16 16 16 8 8 8 8 8 4 4 4 4 4 4 3 3 2 2", "int4": "16 2 2 4 4 4 4 4 4 4", "planes": "p4 p3 p2 4",
         "16": "16", "8": "8", "4": "4", "3": "3", "2": "2"}


def listed():
    return [
        # one token through a square projection at 4 bits
        {"name": "linear_one_token", "op": "linear", "tokens": 1, "cols": 4096, "rows": "4096", "formats": "4", "bias": False, "out": "f16"},
        # queries, keys and values of one token: three blocks at bitwidths of their own, with a bias
        {"name": "linear_three_blocks", "op": "linear", "tokens": 1, "cols": 4096, "rows": "4096,1024,1024", "formats": "4,8,8", "bias": True, "out": "f16"},
        # router logits of a small batch: few and odd rows, a contraction that ends inside a group, 16-bit weights
        {"name": "linear_router_odd", "op": "linear", "tokens": 5, "cols": 2050, "rows": "60", "formats": "16", "bias": False, "out": "f32"},
        # eight tokens through a long contraction, read from overlaid bit-planes at 3 bits
        {"name": "linear_planes", "op": "linear", "tokens": 8, "cols": 14336, "rows": "4096", "formats": "p3", "bias": False, "out": "bf16"},
        # one token over a vocabulary that is no multiple of the page's rows
        {"name": "linear_vocabulary", "op": "linear", "tokens": 1, "cols": 4096, "rows": "32003", "formats": "4", "bias": False, "out": "f32"},
        # a decode batch of 64 through the widest projection
        {"name": "linear_decode", "op": "linear", "tokens": 64, "cols": 4096, "rows": "14336", "formats": "4", "bias": False, "out": "f16"},
        # one token of the smallest layer: all latency
        {"name": "layer_tiny", "op": "layer", "tokens": 1, "experts": 8, "shared": 0, "top_k": 2, "hidden": 256, "ffn": 512, "mix": "mix", "given": False, "padding": 0, "out": "f16"},
        # one token of the 8-expert layer at mixed bitwidths
        {"name": "layer_one_token", "op": "layer", "tokens": 1, "experts": 8, "shared": 0, "top_k": 2, "hidden": 4096, "ffn": 14336, "mix": "mix", "given": False, "padding": 0, "out": "f16"},
        # one token, and four, of the layer with 60 routed and 4 shared experts
        {"name": "layer_one_token_shared", "op": "layer", "tokens": 1, "experts": 60, "shared": 4, "top_k": 4, "hidden": 2048, "ffn": 1408, "mix": "mix", "given": False, "padding": 0, "out": "f16"},
        {"name": "layer_four_tokens_shared", "op": "layer", "tokens": 4, "experts": 60, "shared": 4, "top_k": 4, "hidden": 2048, "ffn": 1408, "mix": "int4", "given": False, "padding": 0, "out": "bf16"},
        # a padded batch of 16 of the layer with many small experts, routed beforehand: the rows of the padding take none
        {"name": "layer_batch_routed", "op": "layer", "tokens": 16, "experts": 128, "shared": 1, "top_k": 8, "hidden": 2048, "ffn": 768, "mix": "int4", "given": True, "padding": 3, "out": "bf16"},
        # eight tokens of the 8-expert layer at 4 bits
        {"name": "layer_batch", "op": "layer", "tokens": 8, "experts": 8, "shared": 0, "top_k": 2, "hidden": 4096, "ffn": 14336, "mix": "4", "given": False, "padding": 0, "out": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.55:
        n = rng.choice((1, 1, 1, 2, 3))
        cols = _log_int(rng, 64, 14336)
        if rng.random() < 0.5:
            cols = _padded(cols)
        most = min(32003, 32003 * 4096 // cols) // n
        rows = [_log_int(rng, 8, most) for _ in range(n)]
        if rng.random() < 0.5:
            rows = [min(_padded(r), max(1, most)) for r in rows]
        return {"op": "linear", "tokens": _log_int(rng, 1, 64), "cols": cols, "rows": ",".join(map(str, rows)),
                "formats": ",".join(rng.choice(("16", "8", "4", "4", "4", "3", "2", "p4", "p3", "p2")) for _ in rows),
                "bias": rng.random() < 0.5, "out": rng.choice(("f16", "bf16", "f32"))}
    hidden = _padded(_log_int(rng, 128, 4096))
    ffn = _padded(_log_int(rng, 128, 14336))
    most = max(2, min(128, 8 * 4096 * 14336 // (hidden * ffn)))
    experts = _log_int(rng, 2, most)
    tokens = _log_int(rng, 1, 16)
    case = {"op": "layer", "tokens": tokens, "experts": experts, "shared": rng.choice((0, 0, 1, 2, 4)) if experts * hidden * ffn < 3 * 4096 * 14336 else 0,
            "top_k": rng.randint(1, min(8, experts)), "hidden": hidden, "ffn": ffn, "mix": rng.choice(("mix", "mix", "int4", "planes", "4", "4", "16", "8", "3", "2")),
            "given": rng.random() < 0.5, "padding": rng.choice((0, 0, 1)) if tokens > 1 else 0, "out": rng.choice(("f16", "bf16"))}
    while work(case)["bytes"] > 650e6:
        case["ffn"] = _padded(case["ffn"] // 2)
    return case


def _padded(n):
    return -(-n // GROUP) * GROUP


def _formats(case):
    """The format of every routed block of a layer, [experts][3]: the mix's shares, dealt out in an order of their own."""
    shares = MIXES[case["mix"]].split()
    n = 3 * case["experts"]
    dealt = [shares[i * len(shares) // n] for i in range(n)] if n >= len(shares) else random.Random(7).sample(shares, n)
    random.Random(3).shuffle(dealt)
    return [dealt[3 * e:3 * e + 3] for e in range(case["experts"])]


# ---- blocks ----------------------------------------------------------------------------------------

class Block:
    """One block as it is stored: codes (a stream of bytes; 16 bits: the weights), scales and zero-points [rows, groups], and,
    for bit-planes, the fp16 weights that the planes are made from."""


def _block(w, fmt):
    """The block of fp16 weights [rows, cols] (multiples of 128) in a format: the codes of a group spread evenly from its
    smallest to its largest weight; read from bit-planes, the first bits of the 4-bit codes, each standing for the middle of
    the levels that it merges."""
    bits, planes = FORMATS[fmt]
    b = Block()
    b.bits, b.planes, b.rows, b.cols, b.weights = bits, planes, w.shape[0], w.shape[1], None
    if bits == 16:
        b.codes, b.scales, b.zeros = w, None, None
        return b
    first = 4 if planes else bits
    v = w.view(b.rows, b.cols // GROUP, GROUP).float()
    lo, hi = v.amin(2, keepdim=True), v.amax(2, keepdim=True)
    scale = ((hi - lo) / (2 ** first - 1)).half()
    scale = torch.where(hi == lo, torch.ones_like(scale), scale.clamp_min(2.0 ** -24))
    codes = torch.round((v - lo) * (1.0 / scale.float())).clamp(0, 2 ** first - 1).to(torch.uint8).view(b.rows, b.cols)
    b.scales, b.zeros = scale.squeeze(2), lo.half().squeeze(2)
    if planes:
        b.weights = w
        merged = 2 ** (4 - bits)
        codes = codes >> (4 - bits)
        b.zeros = (b.zeros.float() + b.scales.float() * ((merged - 1) / 2)).half()
        b.scales = b.scales * merged
    if bits == 8:
        b.codes = codes.view(-1)
    elif bits == 3:
        c = codes.view(-1, 8).int()
        word = (c << (3 * torch.arange(8, device=w.device, dtype=torch.int32))).sum(1)
        b.codes = torch.stack([(word >> (8 * i) & 255).to(torch.uint8) for i in range(3)], 1).view(-1)
    else:
        c = codes.view(-1, 8 // bits)
        b.codes = (c << (bits * torch.arange(8 // bits, device=w.device, dtype=torch.uint8))).sum(1, dtype=torch.uint8)
    return b


def _draw_block(normal, uniform, rows, cols, fmt, padded_rows=None, padded_cols=None):
    """Small weights, one in a thousand ten times larger; what the page has more of is zero."""
    w = normal(rows, cols) * 0.02
    w = torch.where(uniform(rows, cols) < 0.001, w * 10.0, w)
    w = torch.nn.functional.pad(w, (0, (padded_cols or cols) - cols, 0, (padded_rows or rows) - rows)).half()
    return _block(w, fmt)


# ---- inputs ----------------------------------------------------------------------------------------

def prepare(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=d)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=d)

    s = dict(case)
    T = case["tokens"]
    if case["op"] == "linear":
        K, rows = case["cols"], [int(r) for r in case["rows"].split(",")]
        s["n"] = rows
        s["blocks"] = [_draw_block(normal, uniform, r, K, f, _padded(r), _padded(K)) for r, f in zip(rows, case["formats"].split(","))]
        # hidden states behind a norm; rows start 16 bytes apart or a multiple of that
        s["x"] = torch.empty(T, -(-K // 8) * 8, dtype=torch.float16, device=d)[:, :K].copy_(normal(T, K))
        s["bias_t"] = (normal(sum(rows)) * 0.5).half() if case["bias"] else None
        s["out_t"] = torch.empty(T, sum(rows), dtype=TYPES[case["out"]], device=d)
        if own:
            s["pages"] = [_page(_library(), b) for b in s["blocks"]]
        return s
    H, F, E, k = case["hidden"], case["ffn"], case["experts"], case["top_k"]
    formats = _formats(case) + [["16"] * 3] * case["shared"]
    s["blocks"] = [[_draw_block(normal, uniform, *((H, F) if kind == 2 else (F, H)), f) for kind, f in enumerate(three)] for three in formats]
    s["x"] = normal(T, H).half()
    s["logits"] = normal(T, E)
    s["out_t"] = torch.empty(T, H, dtype=TYPES[case["out"]], device=d)
    if case["given"]:                                # a sigmoid router's choice and gates, made before the call
        order = s["logits"].sort(dim=1, descending=True, stable=True).indices[:, :k]
        gates = torch.sigmoid(s["logits"].gather(1, order))
        s["ids"], s["gates"] = order.int(), gates / gates.sum(1, keepdim=True) * 2.5
        s["ids"][T - case["padding"]:] = -1
        s["gates"][T - case["padding"]:] = 0
    if own:
        from paper_2607_16184_b200 import binding
        ctx = s["ctx"] = binding.Context(1, E, case["shared"], H, F, 16, k)
        ctx.pw_set_page_table([(0, e, kind, _page(ctx, b)) for e, three in enumerate(s["blocks"]) for kind, b in enumerate(three)])
    return s


_context = None


def _library():
    """The context that a program keeps for as long as it runs (8 experts of 256 x 512: its workspace is small)."""
    global _context
    from paper_2607_16184_b200 import binding
    if _context is None:
        _context = binding.Context(1, 8, 0, 256, 512, 16, 2)
    return _context


def _page(ctx, b):
    """The library's page of a block."""
    from paper_2607_16184_b200 import binding
    if b.planes:
        return ctx.pw_quantize_planes(b.weights).at(b.bits)
    page = binding.Page(b.rows, b.cols, b.bits, "cuda", binding.PW_LAYOUT_CANONICAL)
    page.codes.copy_(b.codes.contiguous().view(torch.uint8).view(-1))
    if b.bits < 16:
        page.scales.copy_(b.scales.reshape(-1))
        page.zps.copy_(b.zeros.reshape(-1))
    return ctx.pw_import_page(page)


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    s = state
    if own:
        if s["op"] == "linear":
            return {"out": _library().pw_page_linear(s["x"], s["pages"], out_features=s["n"], bias=s["bias_t"], out=s["out_t"])}
        if s["given"]:
            return {"out": s["ctx"].pw_moe_forward_few_routed(0, s["x"], s["ids"], s["gates"], out=s["out_t"])}
        return {"out": s["ctx"].pw_moe_forward_few(0, s["x"], s["logits"], s["top_k"], out=s["out_t"])}
    return {"linear": _linear, "layer": _layer}[s["op"]](s)


def _weights(b, rows=None, cols=None):
    """A block's weights in 32 bits."""
    if b.bits == 16:
        w = b.codes.float()
    else:
        if b.bits == 3:
            three = b.codes.view(-1, 3).int()
            word = three[:, 0] | three[:, 1] << 8 | three[:, 2] << 16
            codes = word[:, None] >> (3 * torch.arange(8, device=word.device, dtype=torch.int32)) & 7
        elif b.bits == 8:
            codes = b.codes
        else:
            codes = b.codes[:, None] >> (b.bits * torch.arange(8 // b.bits, device=b.codes.device, dtype=torch.uint8)) & (2 ** b.bits - 1)
        codes = codes.reshape(b.rows, b.cols // GROUP, GROUP).float()
        w = (codes * b.scales.float()[:, :, None] + b.zeros.float()[:, :, None]).view(b.rows, b.cols)
    return w[:rows, :cols]


def _linear(s):
    x = s["x"].float()
    out = torch.cat([x @ _weights(b, n, s["cols"]).t() for b, n in zip(s["blocks"], s["n"])], 1)
    if s["bias_t"] is not None:
        out = out + s["bias_t"].float()
    return {"out": out.to(TYPES[s["out"]])}


def _layer(s):
    x, E, T = s["x"].float(), s["experts"], s["tokens"]
    if s["given"]:
        ids, gates = s["ids"].long(), s["gates"]
    else:
        order = s["logits"].sort(dim=1, descending=True, stable=True)
        ids = order.indices[:, :s["top_k"]]
        gates = torch.softmax(order.values[:, :s["top_k"]], 1)
    # the gate of every token and expert (shared experts: 1), and the experts that have a token
    share = torch.zeros(T, E + 1, device=x.device).scatter_add_(1, torch.where(ids < 0, E, ids), gates)[:, :E]
    share = torch.cat([share, torch.ones(T, s["shared"], device=x.device)], 1)
    used = ids[ids >= 0].unique().tolist() + list(range(E, E + s["shared"]))
    out = torch.zeros(T, s["hidden"], device=x.device)
    for e in used:
        gate, up, down = s["blocks"][e]
        g = x @ _weights(gate).t()
        h = g / (1.0 + torch.exp(-g)) * (x @ _weights(up).t())
        out += share[:, e, None] * (h @ _weights(down).t())
    return {"out": out.to(TYPES[s["out"]])}


# ---- what a pass cannot do without -----------------------------------------------------------------

def _block_bytes(rows, cols, fmt):
    bits = FORMATS[fmt][0]
    return rows * cols * bits / 8 + (4 * rows * _padded(cols) / GROUP if bits < 16 else 0)


def work(case):
    T = case["tokens"]
    if case["op"] == "linear":
        K, rows = case["cols"], [int(r) for r in case["rows"].split(",")]
        n = sum(_block_bytes(r, K, f) for r, f in zip(rows, case["formats"].split(",")))
        return {"bytes": n + 2 * T * K + T * sum(rows) * SIZE[case["out"]] + (2 * sum(rows) if case["bias"] else 0), "flops": 2 * T * K * sum(rows)}
    H, F, E, k, ns = case["hidden"], case["ffn"], case["experts"], case["top_k"], case["shared"]
    taken = T - case["padding"] if case["given"] else T
    # how many experts get a token, where every choice is as likely: the expected number
    active = E * (1.0 - (1.0 - k / E) ** taken)
    routed = sum(_block_bytes(H, F, f) for three in _formats(case) for f in three) / E
    n = active * routed + ns * 6 * H * F
    return {"bytes": n + T * (2 * H + SIZE[case["out"]] * H + (8 * k if case["given"] else 4 * E)), "flops": 6 * H * F * (taken * k + T * ns)}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _rows64(b, r0, r1, cols):
    """Rows r0 .. r1 of a block in 64 bits, code by code from the bits of the stream."""
    if b.bits == 16:
        return b.codes[r0:r1, :cols].double()
    per = b.cols * b.bits // 8
    stream = b.codes[r0 * per:r1 * per].view(r1 - r0, per)
    at = torch.arange(b.cols, device=stream.device) * b.bits
    code = torch.zeros(r1 - r0, b.cols, dtype=torch.float64, device=stream.device)
    for i in range(b.bits):
        byte = stream[:, (at + i) // 8].int()
        code += torch.remainder(torch.div(byte, 2 ** ((at + i) % 8), rounding_mode="floor"), 2).double() * 2.0 ** i
    for c in range(0, b.cols, GROUP):
        code[:, c:c + GROUP] *= b.scales[r0:r1, c // GROUP, None].double()
        code[:, c:c + GROUP] += b.zeros[r0:r1, c // GROUP, None].double()
    return code[:, :cols]


def _product64(x, b, n=None, cols=None):
    n, step = n or b.rows, 1024
    return torch.cat([x @ _rows64(b, r, min(n, r + step), cols).T for r in range(0, n, step)], 1)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "linear":
        out = torch.cat([_product64(x, b, n, case["cols"]) for b, n in zip(s["blocks"], s["n"])], 1)
        return {"out": out if s["bias_t"] is None else out + s["bias_t"].double()}
    E, k = case["experts"], case["top_k"]
    out = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device=x.device)
    taken = {e: [(t, 1.0) for t in range(case["tokens"])] for e in range(E, E + case["shared"])}
    logits = s["logits"].double().cpu().numpy()
    for t, row in enumerate(logits):
        if case["given"]:
            pairs = list(zip(s["ids"][t].tolist(), s["gates"][t].double().tolist()))
        else:
            best = sorted(range(E), key=lambda e: (-row[e], e))[:k]
            p = np.exp(row[best] - row[best].max())
            pairs = list(zip(best, p / p.sum()))
        for e, gate in pairs:
            if e >= 0:
                taken.setdefault(e, []).append((t, float(gate)))
    for e, rows in taken.items():
        at = torch.tensor([t for t, _ in rows], device=x.device)
        gate, up, down = s["blocks"][e]
        g = _product64(x[at], gate)
        y = _product64(g * torch.sigmoid(g) * _product64(x[at], up), down)
        out.index_add_(0, at, y * torch.tensor([p for _, p in rows], dtype=torch.float64, device=x.device)[:, None])
    return {"out": out}
