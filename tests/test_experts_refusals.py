"""Refusals of the operators for heads that are made of experts, through the C entry points, on the CPU: every bad argument is turned down
before the handle is looked into or anything is launched (the handle here is a block of zeros)."""
import ctypes as C
import os

import pytest

from paper_2505_06641_amd import binding

EINVAL, ECAPACITY, OK = binding.SP_EINVAL, binding.SP_ECAPACITY, binding.SP_OK
P = 1 << 20            # an address with every alignment; nothing reads it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2505_06641_amd import build
        build.build_library(verbose=False)
    return binding.load_library()


@pytest.fixture(scope="module")
def handle():
    return C.cast((C.c_char * 4096)(), C.c_void_p)


def refused(call, base, changes, status=EINVAL):
    for key, value in changes:
        assert key in base
        assert call(*dict(base, **{key: value}).values()) == status, (key, value)


def test_route_refuses(lib, handle):
    base = dict(ops=handle, n=4, experts=8, top=2, dtype=0, z=P, zs=8, score=0, bias=P, groups=2, top_groups=1, renormalize=1, scale=1.0, expert=P,
                weight=P, stream=None)
    refused(lib.sp_route, base, [("ops", None), ("n", -1), ("experts", 0), ("top", 0), ("top", 9), ("top", 5), ("dtype", 2), ("z", None), ("zs", 7),
                                 ("score", 2), ("score", -1), ("groups", 0), ("groups", 3), ("top_groups", 0), ("top_groups", 3), ("scale", float("nan")),
                                 ("scale", float("inf")), ("expert", None), ("weight", None), ("z", P + 2), ("bias", P + 1), ("expert", P + 2),
                                 ("weight", P + 2)])
    assert lib.sp_route(*dict(base, experts=1026, zs=1026).values()) == ECAPACITY
    assert lib.sp_route(*dict(base, experts=64, zs=64, top=33, groups=1).values()) == ECAPACITY
    assert lib.sp_route(*dict(base, experts=130, zs=130, groups=65, top_groups=5).values()) == ECAPACITY
    assert lib.sp_route(*dict(base, dtype=1, z=P + 1).values()) == EINVAL
    assert lib.sp_route(*dict(base, n=0, z=None, expert=None, weight=None).values()) == OK


def test_route_backward_refuses(lib, handle):
    base = dict(ops=handle, n=4, experts=8, top=2, dtype=0, z=P, zs=8, score=0, renormalize=1, scale=1.0, expert=P, dweight=P, dz=P, dzs=8, stream=None)
    refused(lib.sp_route_backward, base, [("ops", None), ("n", -1), ("experts", 0), ("top", 0), ("top", 9), ("dtype", 3), ("z", None), ("zs", 7), ("score", 2),
                                          ("scale", float("inf")), ("expert", None), ("dweight", None), ("dz", None), ("dzs", 7), ("z", P + 2), ("dz", P + 2),
                                          ("expert", P + 1), ("dweight", P + 2)])
    assert lib.sp_route_backward(*dict(base, experts=1025, zs=1025, dzs=1025).values()) == ECAPACITY
    assert lib.sp_route_backward(*dict(base, experts=40, zs=40, dzs=40, top=33).values()) == ECAPACITY
    assert lib.sp_route_backward(*dict(base, n=0).values()) == OK


def test_route_order_refuses(lib, handle):
    base = dict(ops=handle, n=4, top=2, experts=8, expert=P, offsets=P, place=P, stream=None)
    refused(lib.sp_route_order, base, [("ops", None), ("n", -1), ("top", 0), ("experts", 0), ("expert", None), ("offsets", None), ("place", None),
                                       ("expert", P + 2), ("offsets", P + 1), ("place", P + 2)])
    refused(lib.sp_route_order, base, [("top", 33), ("experts", 1025), ("n", 1 << 30)], ECAPACITY)
    # the handle's workspace (0 bytes here) holds no tile's counts
    assert lib.sp_route_order(*dict(base, n=1 << 20).values()) == ECAPACITY


def test_moves_refuse(lib, handle):
    base = dict(ops=handle, n=4, d=8, top=2, dtype=0, x=P, xst=8, place=P, rows=8, xs=P, xss=8, stream=None)
    refused(lib.sp_dispatch, base, [("ops", None), ("n", -1), ("d", 0), ("top", 0), ("dtype", 2), ("x", None), ("xst", 7), ("place", None), ("rows", -1),
                                    ("xs", None), ("xss", 7), ("x", P + 2), ("xs", P + 2), ("place", P + 2)])
    refused(lib.sp_dispatch, base, [("top", 33)], ECAPACITY)
    assert lib.sp_dispatch(*dict(base, d=1 << 21, xst=1 << 21, xss=1 << 21).values()) == ECAPACITY
    assert lib.sp_dispatch(*dict(base, n=0).values()) == OK
    base = dict(ops=handle, n=4, d=8, top=2, dtype=0, rows=8, ys=P, yss=8, place=P, weight=P, r=P, rs=8, y=P, yst=8, stream=None)
    refused(lib.sp_combine, base, [("ops", None), ("n", -1), ("d", 0), ("top", 0), ("dtype", 2), ("rows", -1), ("ys", None), ("yss", 7), ("place", None),
                                   ("rs", 7), ("y", None), ("yst", 7), ("ys", P + 2), ("y", P + 2), ("r", P + 2), ("weight", P + 2), ("place", P + 1)])
    refused(lib.sp_combine, base, [("top", 33)], ECAPACITY)
    assert lib.sp_combine(*dict(base, n=0).values()) == OK
    base = dict(ops=handle, n=4, d=8, top=2, dtype=1, dy=P, dyst=8, rows=8, ys=P, yss=8, place=P, weight=P, dys=P, dyss=8, dweight=P, stream=None)
    refused(lib.sp_combine_backward, base, [("ops", None), ("n", -1), ("d", 0), ("top", 0), ("dtype", 2), ("dy", None), ("dyst", 7), ("rows", -1), ("ys", None),
                                            ("yss", 7), ("place", None), ("dyss", 7), ("dy", P + 1), ("ys", P + 1), ("dys", P + 1), ("weight", P + 2),
                                            ("dweight", P + 2)])
    refused(lib.sp_combine_backward, base, [("top", 33)], ECAPACITY)
    assert lib.sp_combine_backward(*dict(base, dys=None, dweight=None).values()) == OK


def test_dropout_refuses(lib, handle):
    base = dict(ops=handle, n=4, d=8, dtype=0, x=P, xs=8, p=0.5, seed=1, offset=0, step=P, r=P, rs=8, y=P, ys=8, stream=None)
    refused(lib.sp_dropout, base, [("ops", None), ("n", -1), ("d", 0), ("dtype", 2), ("x", None), ("xs", 7), ("p", -0.1), ("p", 1.1), ("p", float("nan")),
                                   ("step", P + 4), ("rs", 7), ("y", None), ("ys", 7), ("x", P + 2), ("y", P + 2), ("r", P + 2)])
    assert lib.sp_dropout(*dict(base, d=1 << 21, xs=1 << 21, ys=1 << 21, rs=1 << 21).values()) == ECAPACITY
    assert lib.sp_dropout(*dict(base, n=0, x=None, y=None).values()) == OK


def test_quantized_refuse(lib, handle):
    base = dict(ops=handle, n=4, d=8, dtype=0, x=P, xs=8, q=P, qs=8, scale=P, stream=None)
    refused(lib.sp_quantize_rows, base, [("ops", None), ("n", -1), ("d", 0), ("dtype", 2), ("x", None), ("xs", 7), ("q", None), ("qs", 7), ("scale", None),
                                         ("x", P + 2), ("scale", P + 2)])
    assert lib.sp_quantize_rows(*dict(base, d=1 << 21, xs=1 << 21, qs=1 << 21).values()) == ECAPACITY
    assert lib.sp_quantize_rows(*dict(base, n=0).values()) == OK
    base = dict(ops=handle, n=4, k=8, m=16, groups=2, x=P, xs=8, x_scale=P, offsets=P, w=P, w_scale=P, bias=P, act=1, out=0, r=P, rs=16, y=P, ys=16, stream=None)
    refused(lib.sp_grouped_linear_quantized, base, [
        ("ops", None), ("n", -1), ("k", 0), ("m", 0), ("groups", 0), ("x", None), ("xs", 7), ("x_scale", None), ("offsets", None), ("w", None), ("w_scale", None),
        ("act", 2), ("out", 2), ("rs", 15), ("y", None), ("ys", 15), ("y", P + 2), ("r", P + 2), ("x_scale", P + 2), ("w_scale", P + 1), ("offsets", P + 2),
        ("bias", P + 2)])
    refused(lib.sp_grouped_linear_quantized, dict(base, xs=1 << 21, ys=1 << 21, rs=1 << 21), [("groups", 65536), ("k", 131072), ("m", (1 << 20) + 1)], ECAPACITY)
    assert lib.sp_grouped_linear_quantized(*dict(base, n=0).values()) == OK
