"""Refusals of the operators around the layer: every one is decided on the host, before a device is touched (CPU only)."""
import ctypes as C

import pytest

from paper_2607_16184_b200 import binding as B
from paper_2607_16184_b200 import build as pwbuild

OK, ARG, SHAPE, ALIGN = 0, 1, 2, 4
P = 1 << 20                                        # an address nobody reads: 16-byte aligned


@pytest.fixture(scope="module")
def lib():
    pwbuild.build()
    return B.load()


@pytest.fixture(scope="module")
def ctx():
    """Stands in for a context: a refused call does not look inside it."""
    return C.create_string_buffer(1 << 16)


def quantize(lib, ctx, x=P, x_type=0, rows=3, cols=40, x_stride=40, block_rows=1, q=P, q_stride=48, scales=P):
    return lib.pw_quantize_scaled(ctx, x, x_type, rows, cols, x_stride, block_rows, q, q_stride, scales, None)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(x=None)), (ARG, dict(q=None)), (ARG, dict(scales=None)), (ARG, dict(x_type=3)), (ARG, dict(x_type=-1)),
    (ARG, dict(rows=-1)), (ARG, dict(cols=0)), (ARG, dict(block_rows=2)), (ARG, dict(block_rows=0)), (SHAPE, dict(x_stride=39)),
    (SHAPE, dict(q_stride=32)), (SHAPE, dict(cols=(1 << 30) + 1)), (ALIGN, dict(q_stride=41)), (ALIGN, dict(x=P + 4)),
    (ALIGN, dict(q=P + 8)), (ALIGN, dict(scales=P + 4)), (OK, dict(rows=0)), (OK, dict(rows=0, x=None, q=None, scales=None))])
def test_quantize_refuses(lib, ctx, status, change):
    assert quantize(lib, ctx, **change) == status


def norm(lib, ctx, T=2, H=40, x=P, x_type=0, x_stride=40, r=P, r_type=1, r_stride=40, w=P, w_type=1, eps=1e-6, ro=P, ro_stride=40,
         y=P, y_type=1, y_stride=40, q=P, q_stride=48, qs=P):
    return lib.pw_add_rmsnorm(ctx, T, H, x, x_type, x_stride, r, r_type, r_stride, w, w_type, eps, ro, ro_stride, y, y_type, y_stride,
                              q, q_stride, qs, None)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(x=None)), (ARG, dict(w=None)), (ARG, dict(y=None, q=None, qs=None)), (ARG, dict(q=None)), (ARG, dict(qs=None)),
    (ARG, dict(r=None)), (ARG, dict(x_type=7)), (ARG, dict(r_type=3)), (ARG, dict(w_type=3)), (ARG, dict(y_type=-1)),
    (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(T=-1)), (ARG, dict(H=0)), (SHAPE, dict(H=32769)),
    (SHAPE, dict(x_stride=39)), (SHAPE, dict(r_stride=39)), (SHAPE, dict(ro_stride=39)), (SHAPE, dict(y_stride=39)),
    (SHAPE, dict(q_stride=32)), (ALIGN, dict(q_stride=44)), (ALIGN, dict(x=P + 4)), (ALIGN, dict(r=P + 2)), (ALIGN, dict(w=P + 2)),
    (ALIGN, dict(ro=P + 2)), (ALIGN, dict(y=P + 2)), (ALIGN, dict(q=P + 1)), (ALIGN, dict(qs=P + 4)),
    (OK, dict(T=0, x=None, w=None, r=None, ro=None, y=None, q=None, qs=None))])
def test_norm_refuses(lib, ctx, status, change):
    assert norm(lib, ctx, **change) == status


def linear(lib, ctx, T=2, N=24, K=40, a=P, a_stride=48, sa=P, w=P, w_stride=48, sw=P, out=P, out_type=1, out_stride=24):
    return lib.pw_scaled_linear(ctx, T, N, K, a, a_stride, sa, w, w_stride, sw, out, out_type, out_stride, None)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(a=None)), (ARG, dict(sa=None)), (ARG, dict(w=None)), (ARG, dict(sw=None)), (ARG, dict(out=None)), (ARG, dict(out_type=5)),
    (ARG, dict(T=-1)), (ARG, dict(N=0)), (ARG, dict(K=0)), (SHAPE, dict(a_stride=32)), (SHAPE, dict(w_stride=32)),
    (SHAPE, dict(out_stride=23)), (SHAPE, dict(N=(1 << 30) + 1)), (SHAPE, dict(K=(1 << 30) + 1)), (ALIGN, dict(a_stride=40)),
    (ALIGN, dict(w_stride=52)), (ALIGN, dict(a=P + 8)), (ALIGN, dict(w=P + 4)), (ALIGN, dict(sa=P + 4)), (ALIGN, dict(sw=P + 4)),
    (ALIGN, dict(out=P + 2)), (OK, dict(T=0)), (OK, dict(T=0, a=None, out=None))])
def test_linear_refuses(lib, ctx, status, change):
    assert linear(lib, ctx, **change) == status


def route(lib, ctx, E=16, k=2, score=0, groups=4, top=2, best=1, renorm=1, scale=1.0, logits=P, t=0, stride=16, bias=None, T=3,
          ids=P, gates=P, rule=True):
    r = B.pw_routing(E, k, score, groups, top, best, renorm, scale)
    return lib.pw_route_tokens(ctx, C.byref(r) if rule else None, logits, t, stride, bias, T, ids, gates, None)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(rule=False)), (ARG, dict(E=0)), (ARG, dict(E=257, groups=1, top=1, stride=257)), (ARG, dict(k=0)), (ARG, dict(k=9)),
    (ARG, dict(E=64, k=33, top=4)), (ARG, dict(score=2)), (ARG, dict(groups=0)), (ARG, dict(groups=3)), (ARG, dict(groups=32)),
    (ARG, dict(top=0)), (ARG, dict(top=5)), (ARG, dict(best=0)), (ARG, dict(best=3)), (ARG, dict(scale=float("nan"))),
    (ARG, dict(scale=float("inf"))), (ARG, dict(logits=None)), (ARG, dict(ids=None)), (ARG, dict(gates=None)), (ARG, dict(t=3)),
    (ARG, dict(T=-1)), (SHAPE, dict(stride=15)), (ALIGN, dict(logits=P + 4)), (ALIGN, dict(bias=P + 4)), (ALIGN, dict(ids=P + 4)),
    (ALIGN, dict(gates=P + 8)), (OK, dict(T=0)), (OK, dict(T=0, logits=None, ids=None, gates=None))])
def test_route_refuses(lib, ctx, status, change):
    assert route(lib, ctx, **change) == status


def test_null_context(lib):
    assert quantize(lib, None) == norm(lib, None) == linear(lib, None) == route(lib, None) == ARG
    assert lib.pw_moe_forward_routed(None, 0, P, P, P, 1, 1, None, P, 0, None) == ARG
