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
