"""Refusals of the calls for few tokens that are decided before a context or a device is looked at (CPU only)."""
import ctypes as C

import pytest

from paper_2607_16184_b200 import binding as B
from paper_2607_16184_b200 import build as pwbuild

OK, ARG, SHAPE, BITS, ALIGN, STATE = 0, 1, 2, 3, 4, 5
P = 1 << 20                                        # an address nobody reads: 16-byte aligned


@pytest.fixture(scope="module")
def lib():
    pwbuild.build()
    return B.load()


@pytest.fixture(scope="module")
def ctx():
    """Stands in for a context: a refused call does not look inside it."""
    return C.create_string_buffer(1 << 16)


def page(codes=P, scales=None, zps=None, rows=256, cols=256, group=128, bits=4, layout=B.PW_LAYOUT_TILED):
    return B.pw_page(codes, scales, zps, rows, cols, group, bits, layout)


def linear(lib, ctx, T=2, K=200, x=P, x_stride=200, pages=None, n=None, n_pages=None, bias=None, bias_type=0, out=P, out_type=1, out_stride=512, workspace=None):
    pages = [page()] if pages is None else pages
    a = (B.pw_page * max(1, len(pages)))(*pages)
    f = None if n is None else (C.c_int32 * len(n))(*n)
    return lib.pw_page_linear(ctx, T, K, x, x_stride, a if pages else None, f, len(pages) if n_pages is None else n_pages, bias, bias_type, out,
                              out_type, out_stride, workspace, 0, None)


PLANES = B.PW_LAYOUT_PLANES


@pytest.mark.parametrize("status,change", [
    (ARG, dict(T=-1)), (ARG, dict(K=0)), (ARG, dict(pages=[])), (ARG, dict(n_pages=0)), (ARG, dict(pages=[page()] * 9)), (ARG, dict(x=None)),
    (ARG, dict(out=None)), (ARG, dict(out_type=3)), (ARG, dict(bias=P, bias_type=-1)), (ARG, dict(n=[0])), (ARG, dict(pages=[page(codes=None)])),
    (SHAPE, dict(T=(1 << 24) + 1)), (SHAPE, dict(K=257)), (SHAPE, dict(K=128)), (SHAPE, dict(n=[257])), (SHAPE, dict(pages=[page(rows=250)])),
    (SHAPE, dict(pages=[page(cols=250)])), (SHAPE, dict(pages=[page(group=64)])), (SHAPE, dict(pages=[page(), page(cols=384)])),
    (SHAPE, dict(pages=[page(rows=0)])), (SHAPE, dict(x_stride=199)), (SHAPE, dict(out_stride=255)), (SHAPE, dict(pages=[page()] * 2, out_stride=511)),
    (SHAPE, dict(K=(1 << 18) + 100, x_stride=1 << 20, pages=[page(cols=(1 << 18) + 128)])),
    (BITS, dict(pages=[page(bits=5)])), (BITS, dict(pages=[page(bits=8, layout=PLANES)])), (BITS, dict(pages=[page(bits=16, layout=PLANES)])),
    (STATE, dict(pages=[page(layout=B.PW_LAYOUT_CANONICAL)])), (STATE, dict(pages=[page(bits=3, layout=PLANES)])),
    (STATE, dict(pages=[page(bits=4, scales=P, layout=PLANES)])), (ALIGN, dict(x=P + 8)), (ALIGN, dict(x_stride=204)), (ALIGN, dict(out=P + 4)),
    (ALIGN, dict(bias=P + 4)), (ALIGN, dict(workspace=P + 16)), (ALIGN, dict(pages=[page(codes=P + 8)])), (ALIGN, dict(pages=[page(bits=3, scales=P + 8, layout=PLANES)])),
    (OK, dict(T=0)), (OK, dict(T=0, x=None, out=None)), (OK, dict(T=0, pages=[page(bits=2, layout=PLANES)] * 8, n=[1] * 8))])
def test_page_linear_refuses(lib, ctx, status, change):
    assert linear(lib, ctx, **change) == status


def test_null_context_and_output_type(lib, ctx):
    assert linear(lib, None) == ARG
    assert lib.pw_moe_forward_few(None, 0, P, P, 1, 1, None, P, 0, None) == ARG
    assert lib.pw_moe_forward_few_routed(None, 0, P, P, P, 1, 1, None, P, 0, None) == ARG
    assert lib.pw_moe_forward_few(ctx, 0, P, P, 1, 1, None, P, 3, None) == ARG
    assert lib.pw_moe_forward_few_routed(ctx, 0, P, P, P, 1, 1, None, P, -1, None) == ARG
