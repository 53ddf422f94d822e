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
