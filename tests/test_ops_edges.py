"""The operators that train the heads where their contract is easily missed: ends of the ranges, values that are no numbers, empty
batches, tensors that change under a caller's list."""
import math

import numpy as np
import pytest

from paper_2505_06641_amd import binding
from tests.test_ops import DEV, U, assert_within, dtype_of, gpu, half_step, offsets_of, ops, plain_linear, plain_linear_backward
from tests.test_ops_refusals import P, handle, lib

INT_MAX = 2 ** 31 - 1


@pytest.mark.gpu
def test_loss_of_the_widest_row_stays_inside_it(gpu, ops):
    """One row of 2^31 - 1 classes, even odds, its gradient in the logits' place, between guards wider than the kernel's step."""
    torch, _ = gpu
    guard = 1 << 14
    store = torch.full((2 * guard + INT_MAX,), 7.0, dtype=torch.bfloat16, device=DEV)
    row = store[guard:guard + INT_MAX].view(1, INT_MAX)
    row.zero_()
    label = torch.tensor([INT_MAX - 1], dtype=torch.int32, device=DEV)
    loss = torch.full((1,), math.nan, device=DEV)
    ops.sp_cross_entropy(row, label, loss, dlogits=row)
    # terms of 1 add up exactly; the logarithm and the exponential are off by a few u
    want = math.log(INT_MAX)
    assert abs(float(loss) - want) <= 8 * U * want
    assert bool((store[:guard] == 7).all()) and bool((store[guard + INT_MAX:] == 7).all())
    assert float(row[0, -1]) == -1.0
    first = float(row[0, 0])
    assert abs(first * INT_MAX - 1) <= half_step(torch, torch.bfloat16) + 8 * U
    step = 1 << 28
    for lo in range(0, INT_MAX - 1, step):
        assert bool((row[0, lo:min(lo + step, INT_MAX - 1)] == first).all())


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
def test_a_list_of_gradients_finds_them_where_they_are(gpu, ops, in_place):
    """Tensors of a list that get other storage, another size or another type after it was made."""
    torch, binding = gpu
    grads = [torch.randn(1000, device=DEV), torch.randn(20, 3, device=DEV), torch.randn(0, device=DEV)]
    outs = None if in_place else [torch.zeros_like(g) for g in grads]
    made = binding.TensorList(grads, out=outs)
    norm = torch.empty(1, device=DEV)
    held = [t.data for t in grads + (outs or [])]            # the old values' memory lives on, and stays as it is
    was = [t.clone() for t in held]

    def clipped():
        want = [g.double() for g in grads]
        size = math.sqrt(sum(float((g * g).sum()) for g in want))
        ops.sp_clip_grad_norm(made, 0.5, norm)
        # the norm is rounded once; factor and product once each
        assert abs(float(norm) - size) <= 2 * U * size
        for got, g in zip(outs or grads, want):
            bound = 4 * U * g.abs() + 1e-40
            assert_within(torch, got, g * min(1.0, 0.5 / (size + 1e-6)), bound, "clipped")

    for g in grads:
        g.data = torch.randn_like(g)
    for o in outs or []:
        o.data = torch.full_like(o, math.nan)
    clipped()
    for old, values in zip(held, was):
        assert torch.equal(old, values)
    for t in [grads[0]] + (outs or [])[:1]:                   # longer than what was there
        t.data = torch.randn(50_000, device=DEV)
    clipped()
    good = grads[1].data
    for other in (good.bfloat16(), good.cpu(), torch.randn(6, 20, device=DEV).t()[:, ::2]) + (() if in_place else (torch.randn(5, device=DEV),)):
        grads[1].data = other
        with pytest.raises(binding.SneakPeekError) as e:
            ops.sp_clip_grad_norm(made, 0.5, norm)
        assert e.value.status == binding.SP_EINVAL
    grads[1].data = good
    clipped()


# rows of the groups, inputs, outputs: dx and dW in one launch, dx of few rows apart from dW, tiles of 128 rows, narrow tiles
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,m", [((40, 60), 24, 20), ((3, 2) * 35, 200, 700), ((4100, 5000), 300, 260), ((9000, 3000), 64, 64)])
def test_gradients_pass_where_the_activation_is_above_zero(gpu, ops, sizes, k, m, dtype):
    """NaN, infinities and both zeros among the activations."""
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    g = torch.Generator(device=DEV).manual_seed(3)
    n = sum(sizes)
    x, dy, act = (torch.randn(n, w, device=DEV, generator=g).to(t) for w in (k, m, m))
    a = len(sizes)
    w = (torch.randn(a, k, m, device=DEV, generator=g) / math.sqrt(k)).to(t)
    act[::3, ::2] = math.nan
    act[1::7, 1] = math.inf
    act[2::7, 1] = -math.inf
    act[::5, 3] = 0.0
    act[1::5, 3] = -0.0
    dy[act.isnan() & (torch.rand(n, m, device=DEV, generator=g) < 0.5)] = math.nan       # nothing of these is left either
    dx, dw, db = torch.empty_like(x), torch.empty(a, k, m, device=DEV), torch.empty(a, m, device=DEV)
    offsets = offsets_of(torch, sizes)
    ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, dx=dx, dw=dw, db=db)
    wx, ww, wb, sx, sw, sb = plain_linear_backward(torch, dy, act, x, sizes, w)
    bound = (m + 10) * U * sx
    assert_within(torch, dx, wx, bound + half_step(torch, t) * (wx.abs() + bound), "dx")
    rows = (max(sizes) + 10) * U
    assert_within(torch, dw, ww, rows * sw, "dw")
    assert_within(torch, db, wb, rows * sb, "db")
    ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, db=db.fill_(math.nan))
    assert_within(torch, db, wb, rows * sb, "db alone")


@pytest.mark.gpu
def test_loss_without_rows(gpu, ops):
    torch, _ = gpu
    i = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    z, none = torch.empty(0, 5, device=DEV), torch.empty(0, device=DEV)
    ops.sp_cross_entropy(z, i(0), none, app=i(0), n_classes=i(3) + 5, weight=none.clone(), dlogits=z.clone())
    ops.sp_cross_entropy(z, i(0), none)


def test_loss_without_rows_takes_an_app_array_without_an_address(lib, handle):
    base = dict(ops=handle, n=0, c=8, dtype=0, z=None, zs=8, apps=2, app=None, n_classes=P, label=None, weight=None, scale=1.0, loss=None, gt=0,
                dz=None, dzs=8, stream=None)
    assert lib.sp_cross_entropy(*base.values()) == binding.SP_OK
    assert lib.sp_cross_entropy(*dict(base, app=P).values()) == binding.SP_OK
    assert lib.sp_cross_entropy(*dict(base, app=P, n_classes=None).values()) == binding.SP_EINVAL
    assert lib.sp_cross_entropy(*dict(base, app=P, apps=0).values()) == binding.SP_EINVAL
    assert lib.sp_cross_entropy(*dict(base, n=1, z=P, label=P, loss=P, dz=P).values()) == binding.SP_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,m", [(262144, 64), (200003, 5), (1025, 70)])
def test_bias_gradient_alone_of_long_groups(gpu, ops, n, m, dtype):
    """Equal values, whose roundings in one long sum all go the same way, and random ones."""
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    g = torch.Generator(device=DEV).manual_seed(n + m)
    x, w = torch.zeros(n, 1, dtype=t, device=DEV), torch.zeros(1, 1, m, dtype=t, device=DEV)
    offsets = offsets_of(torch, (n,))
    act = torch.randn(n, m, device=DEV, generator=g).to(t)
    for dy in (torch.full((n, m), 0.1, dtype=t, device=DEV), torch.randn(n, m, device=DEV, generator=g).to(t)):
        for mask in (None, act):
            db = torch.full((1, m), math.nan, device=DEV)
            ops.sp_grouped_linear_backward(dy, x, offsets, w, act=mask, db=db)
            dz = dy.double() if mask is None else torch.where(mask > 0, dy.double(), 0.0)
            # a thread's 256 rows, its n / 1024 parts, four threads
            bound = (256 + math.ceil(n / 1024) + 4) * U * dz.abs().sum(0)[None]
            assert_within(torch, db, dz.sum(0)[None], bound, "db")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_rows_of_the_most_applications(gpu, ops, dtype):
    """Five rows of 65535 applications with wide layers: no more workgroups than rows can fill."""
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    g = torch.Generator(device=DEV).manual_seed(1)
    apps, k, m = 65535, 1, 4096
    w = torch.randn(apps, k, m, device=DEV, generator=g).to(t)
    x = torch.randn(6, k, device=DEV, generator=g).to(t)
    owner = [0, 3, 3, 40000, 65534]                           # the sixth row is of no application
    counts = torch.bincount(torch.tensor(owner), minlength=apps)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).int().to(DEV)
    y = torch.full((6, m), math.nan, dtype=t, device=DEV)
    ops.sp_grouped_linear(x, offsets, w, y)
    want = x[:5].double() * w[owner, 0].double()
    bound = (k + 10) * U * want.abs()
    assert_within(torch, y[:5], want, bound + half_step(torch, t) * (want.abs() + bound), "y")
    assert not y[5].any()
    dy = torch.randn(6, m, device=DEV, generator=g).to(t)
    dx = torch.full((6, k), math.nan, dtype=t, device=DEV)
    ops.sp_grouped_linear_backward(dy, x, offsets, w, dx=dx)
    terms = dy[:5].double() * w[owner, 0].double()
    bound = (m + 10) * U * terms.abs().sum(1, keepdim=True)
    want = terms.sum(1, keepdim=True)
    assert_within(torch, dx[:5], want, bound + half_step(torch, t) * (want.abs() + bound), "dx")
    assert not dx[5].any()


def test_launches_beyond_32_bits_of_threads_are_refused(lib, handle):
    """2^24 tiles of 256 threads, 2^23 of 512 (a mask): more than a launch counts."""
    forward = dict(ops=handle, n=INT_MAX, k=1, m=1, groups=1, dtype=1, x=P, xs=1, offsets=P, w=P, bias=None, act=0, out=1, r=None, rs=1, y=P, ys=1,
                   act_out=None, acts=1, stream=None)
    assert lib.sp_grouped_linear(*forward.values()) == binding.SP_ECAPACITY
    back = dict(ops=handle, n=INT_MAX, k=1, m=1, groups=1, dtype=1, dy=P, dys=1, act=None, acts=1, x=P, xs=1, offsets=P, w=P, dx=P, dxs=1, dw=None,
                db=None, stream=None)
    assert lib.sp_grouped_linear_backward(*back.values()) == binding.SP_ECAPACITY
    masked = dict(back, n=1 << 30, k=65, xs=65, dxs=65, act=P)
    assert lib.sp_grouped_linear_backward(*masked.values()) == binding.SP_ECAPACITY


def test_the_check_waits_for_the_current_stream_of_the_operators_device(lib, monkeypatch):
    """As the other calls do; the device of the program may be another one."""
    import types

    import torch
    kind = binding._ops_class()
    o = kind.__new__(kind)
    o.device, o.h, seen = 1, None, []
    o.lib = types.SimpleNamespace(sp_ops_check=lambda h, stream: seen.append(stream) or binding.SP_OK)
    stream_of = {None: 10, 0: 10, 1: 11}
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=stream_of[device]))
    monkeypatch.setattr(binding, "_current_stream", lambda: 10)
    o.sp_ops_check()
    o.sp_ops_check(stream=types.SimpleNamespace(cuda_stream=12))
    assert seen == [11, 12]


# y and dx of few rows, and in tiles
@pytest.mark.gpu
@pytest.mark.parametrize("n,k,m", [(40, 32, 48), (6000, 300, 600)])
@pytest.mark.parametrize("power", [-60, -100, -110, -114, -118, -122, -126, -130])
def test_small_float32_factors(gpu, ops, n, k, m, power):
    """Factors of 2^power, which a third bfloat16 number cannot finish below 2^-110, against ordinary ones."""
    torch, _ = gpu
    g = torch.Generator(device=DEV).manual_seed(-power)
    small = lambda *s: torch.randn(*s, device=DEV, generator=g) * 2.0 ** power
    offsets = offsets_of(torch, (n,))
    x, w = small(n, k), torch.randn(1, k, m, device=DEV, generator=g)

    def bound(terms, left, right):
        """left @ right: the float32 sum and what the split leaves out, what is left over of either factor, products below 2^-149."""
        a, b = left.double().abs(), right.double().abs()
        over = 2.0 ** -134 * (a.sum(1)[:, None] + b.sum(0)[None])
        return (terms + 10) * U * (a @ b) + over + 6 * terms * 2.0 ** -149

    y = torch.full((n, m), math.nan, device=DEV)
    ops.sp_grouped_linear(x, offsets, w, y)
    assert_within(torch, y, x.double() @ w[0].double(), bound(k, x, w[0]), "y")
    dy, r = small(n, m), torch.randn(n, k, device=DEV, generator=g)
    dx, dw, db = torch.full((n, k), math.nan, device=DEV), torch.full((1, k, m), math.nan, device=DEV), torch.full((1, m), math.nan, device=DEV)
    ops.sp_grouped_linear_backward(dy, r, offsets, w, dx=dx, dw=dw, db=db)
    wt, rt = w[0].t().contiguous(), r.t().contiguous()
    assert_within(torch, dx, dy.double() @ wt.double(), bound(m, dy, wt), "dx")
    assert_within(torch, dw[0], rt.double() @ dy.double(), bound(n, rt, dy), "dw")
    assert_within(torch, db[0], dy.double().sum(0), (n + 8) * U * dy.double().abs().sum(0) + n * 2.0 ** -149, "db")


def test_the_split_of_float32_on_the_host():
    """Three bfloat16 numbers, each the rounded rest, are the value from 2^-110 on; what the three smallest products come to."""
    import torch
    g = torch.Generator().manual_seed(0)
    v = torch.randn(1 << 16, generator=g) * torch.exp2(torch.randint(-100, 100, (1 << 16,), generator=g).float())
    v = torch.cat([v, torch.tensor([1.0038986, 1 + 2.0 ** -8, 1 + 2.0 ** -8 - 2.0 ** -23, 2 - 2.0 ** -23, 2.0 ** -110])])

    def split(q):
        parts = []
        for _ in range(3):
            parts.append(q.bfloat16().float())
            q = q - parts[-1]
        return parts, q

    (a, b, c), rest = split(v)
    assert not rest.any()
    assert bool((b.abs() <= 2.0 ** -8 * v.abs()).all()) and bool((c.abs() <= 2.0 ** -17 * v.abs()).all())
    u = v.roll(7)
    (_, d, e), _ = split(u)
    left_out = (b.double() * e.double()).abs() + (c.double() * d.double()).abs() + (c.double() * e.double()).abs()
    assert bool((left_out <= 2.0 ** -24 * (1 + 2.0 ** -10) * (v.double() * u.double()).abs()).all())
    tiny = v.sign() * torch.rand(v.shape, generator=g) * 2.0 ** -110
    assert bool((split(tiny)[1].abs() <= 2.0 ** -134).all())
