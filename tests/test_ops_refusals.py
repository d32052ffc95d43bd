"""Refusals of the operators that train the heads, through the C entry points, on the CPU: every bad argument is turned down
before the handle is looked into or anything is launched (the handle here is a block of zeros)."""
import ctypes as C
import os

import pytest

from paper_2505_06641_amd import binding

EINVAL, ECAPACITY, EDEVICE = binding.SP_EINVAL, binding.SP_ECAPACITY, binding.SP_EDEVICE
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


def calls(base, changes):
    """(name, arguments) of the call with one argument changed at a time."""
    for key, value in changes:
        args = dict(base)
        args[key] = value
        yield f"{key}={value}", list(args.values())


def test_create_refuses(lib):
    h = C.c_void_p()
    assert lib.sp_ops_create(0, 1 << 20, None) == EINVAL
    assert lib.sp_ops_create(0, (1 << 20) - 1, C.byref(h)) == EINVAL and h.value is None
    assert lib.sp_ops_create(0, -1, C.byref(h)) == EINVAL
    assert lib.sp_ops_create(-1, 1 << 20, C.byref(h)) == EDEVICE and h.value is None
    assert lib.sp_ops_create(10000, 1 << 20, C.byref(h)) == EDEVICE
    lib.sp_ops_destroy(None)
    assert lib.sp_ops_check(None, None) == EINVAL
    assert lib.sp_ops_last_hip_error(None) == b""


def test_layer_norm_refuses(lib, handle):
    base = dict(ops=handle, n=4, d=8, dtype=0, x=P, xs=8, gamma=P, beta=P, eps=1e-5, y=P, ys=8, mean=P, rstd=P, stream=None)
    changes = [("ops", None), ("n", -1), ("d", 0), ("dtype", 2), ("dtype", -1), ("x", None), ("xs", 7), ("eps", -1.0), ("eps", float("nan")),
               ("eps", float("inf")), ("y", None), ("ys", 7), ("x", P + 2), ("y", P + 1), ("gamma", P + 2), ("beta", P + 2),
               ("mean", P + 1), ("rstd", P + 3)]
    for what, args in calls(base, changes):
        assert lib.sp_layer_norm(*args) == EINVAL, what
    wide = dict(base, d=16385, xs=16385, ys=16385)
    assert lib.sp_layer_norm(*wide.values()) == ECAPACITY
    assert lib.sp_layer_norm(*dict(base, dtype=1, x=P + 1).values()) == EINVAL
    assert lib.sp_layer_norm(*dict(base, n=0, x=None, y=None).values()) == binding.SP_OK


def test_layer_norm_backward_refuses(lib, handle):
    base = dict(ops=handle, n=4, d=8, dtype=0, dy=P, dys=8, x=P, xs=8, gamma=P, mean=P, rstd=P, dx=P, dxs=8, dgamma=P, dbeta=P, stream=None)
    changes = [("ops", None), ("n", -1), ("d", 0), ("dtype", 5), ("dy", None), ("dys", 7), ("x", None), ("xs", 7), ("mean", None),
               ("rstd", None), ("dxs", 7), ("dx", P + 1), ("dgamma", P + 2), ("dbeta", P + 2), ("dy", P + 2), ("gamma", P + 1)]
    for what, args in calls(base, changes):
        assert lib.sp_layer_norm_backward(*args) == EINVAL, what
    assert lib.sp_layer_norm_backward(*dict(base, d=16385, dys=16385, xs=16385, dxs=16385).values()) == ECAPACITY
    assert lib.sp_layer_norm_backward(*dict(base, dx=None, dgamma=None, dbeta=None).values()) == binding.SP_OK


def test_grouped_linear_refuses(lib, handle):
    base = dict(ops=handle, n=4, k=8, m=16, groups=2, dtype=0, x=P, xs=8, offsets=P, w=P, bias=P, act=1, out=0, r=P, rs=16, y=P, ys=16,
                act_out=P, acts=16, stream=None)
    changes = [("ops", None), ("n", -1), ("k", 0), ("m", 0), ("groups", 0), ("dtype", 2), ("x", None), ("xs", 7), ("offsets", None),
               ("w", None), ("act", 2), ("act", -1), ("out", 1), ("out", 3), ("rs", 15), ("y", None), ("ys", 15), ("acts", 15), ("x", P + 2),
               ("w", P + 2), ("y", P + 2), ("r", P + 2), ("act_out", P + 2), ("offsets", P + 2), ("bias", P + 2)]
    for what, args in calls(base, changes):
        assert lib.sp_grouped_linear(*args) == EINVAL, what
    assert lib.sp_grouped_linear(*dict(base, groups=65536).values()) == ECAPACITY
    assert lib.sp_grouped_linear(*dict(base, k=(1 << 20) + 1).values()) == ECAPACITY
    assert lib.sp_grouped_linear(*dict(base, m=(1 << 20) + 1).values()) == ECAPACITY
    assert lib.sp_grouped_linear(*dict(base, n=0).values()) == binding.SP_OK


def test_grouped_linear_backward_refuses(lib, handle):
    base = dict(ops=handle, n=4, k=8, m=16, groups=2, dtype=1, dy=P, dys=16, act=P, acts=16, x=P, xs=8, offsets=P, w=P, dx=P, dxs=8, dw=P,
                db=P, stream=None)
    changes = [("ops", None), ("n", -1), ("k", 0), ("m", 0), ("groups", 0), ("dtype", 2), ("dy", None), ("dys", 15), ("acts", 15),
               ("x", None), ("xs", 7), ("offsets", None), ("w", None), ("dxs", 7), ("dy", P + 1), ("act", P + 1), ("x", P + 1), ("w", P + 1),
               ("dx", P + 1), ("dw", P + 2), ("db", P + 2)]
    for what, args in calls(base, changes):
        assert lib.sp_grouped_linear_backward(*args) == EINVAL, what
    assert lib.sp_grouped_linear_backward(*dict(base, groups=65536).values()) == ECAPACITY
    assert lib.sp_grouped_linear_backward(*dict(base, dx=None, dw=None, db=None).values()) == binding.SP_OK


def test_cross_entropy_refuses(lib, handle):
    base = dict(ops=handle, n=4, c=8, dtype=0, z=P, zs=8, apps=2, app=P, n_classes=P, label=P, weight=P, scale=1.0, loss=P, gt=0, dz=P, dzs=8,
                stream=None)
    changes = [("ops", None), ("n", -1), ("c", 0), ("dtype", 2), ("z", None), ("zs", 7), ("apps", 0), ("app", None), ("n_classes", None),
               ("label", None), ("scale", float("nan")), ("scale", float("inf")), ("loss", None), ("gt", 2), ("dzs", 7), ("z", P + 2),
               ("dz", P + 2), ("app", P + 2), ("label", P + 1), ("weight", P + 2), ("loss", P + 2)]
    for what, args in calls(base, changes):
        assert lib.sp_cross_entropy(*args) == EINVAL, what
    assert lib.sp_cross_entropy(*dict(base, dtype=1, gt=0).values()) == EINVAL      # a float32 gradient of bfloat16 logits
    assert lib.sp_cross_entropy(*dict(base, n=0).values()) == binding.SP_OK


def test_clip_refuses(lib, handle):
    ptr = lambda *v: (C.c_void_p * len(v))(*v)
    size = lambda *v: (C.c_int64 * len(v))(*v)
    base = dict(ops=handle, n=2, dtype=0, grads=ptr(P, P), sizes=size(4, 4), max_norm=1.0, out=ptr(P, P), norm=P, stream=None)
    changes = [("ops", None), ("n", -1), ("dtype", 2), ("grads", None), ("sizes", None), ("max_norm", -1.0), ("max_norm", float("nan")),
               ("max_norm", float("inf")), ("norm", None), ("norm", P + 2), ("grads", ptr(P, None)), ("grads", ptr(P, P + 2)),
               ("out", ptr(None, P)), ("out", ptr(P, P + 1)), ("sizes", size(4, -1))]
    for what, args in calls(base, changes):
        assert lib.sp_clip_grad_norm(*args) == EINVAL, what
    # the handle's workspace (0 bytes here) is too small for any tensor's sums
    assert lib.sp_clip_grad_norm(*base.values()) == ECAPACITY
    assert lib.sp_clip_grad_norm(*dict(base, sizes=size(1 << 45, 4)).values()) == ECAPACITY


def test_row_strides_beyond_what_a_tile_reaches_are_refused(lib, handle):
    forward = dict(ops=handle, n=4, k=8, m=16, groups=2, dtype=0, x=P, xs=1 << 24, offsets=P, w=P, bias=P, act=1, out=0, r=P, rs=16, y=P, ys=16,
                   act_out=P, acts=16, stream=None)
    assert lib.sp_grouped_linear(*forward.values()) == ECAPACITY
    back = dict(ops=handle, n=4, k=8, m=16, groups=2, dtype=1, dy=P, dys=16, act=P, acts=16, x=P, xs=8, offsets=P, w=P, dx=P, dxs=8, dw=P,
                db=P, stream=None)
    for key in ("dys", "acts", "xs"):
        assert lib.sp_grouped_linear_backward(*dict(back, **{key: 1 << 24}).values()) == ECAPACITY, key
