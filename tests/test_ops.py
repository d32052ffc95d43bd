"""The operators that train the heads against their definitions in 64 bits, on the GPU.

Tolerances.  u = 2^-24 is half a step of float32, `half_step` that of the output's type.  A sum of t products in float32, in
whatever order and with products whose factors are split exactly, is off by at most (t + 8) u times the sum of the magnitudes; what
is computed from sums of a row carries the sums' relative error and a few u of its own.  Each bound is written out where it is used.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    from paper_2505_06641_amd import binding
    binding.load_library()
    return torch, binding


@pytest.fixture(scope="module")
def ops(gpu):
    o = gpu[1].Ops()
    yield o
    o.sp_ops_check()
    o.close()


def half_step(torch, t):
    return torch.finfo(t).eps / 2


def dtype_of(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def make_rows(torch, rng, n, d, t, layout, scale=1.0):
    """[n, d] values in one of three layouts: contiguous, rows further apart than they are long, and rows that start at addresses
    with no more alignment than an element's."""
    v = torch.from_numpy(rng.standard_normal((n, d)) * scale).to(t)
    if layout == "plain":
        return v.to(DEV)
    pad, lead = {"apart": (16, 0), "odd": (3, 1)}[layout]
    store = torch.full((n * (d + pad) + lead + 1,), float("nan"), dtype=t, device=DEV)
    out = store[lead:lead + n * (d + pad)].view(n, d + pad)[:, :d]
    out.copy_(v)
    return out


def empty_rows(torch, n, d, t, layout):
    return make_rows(torch, np.random.default_rng(0), n, d, t, layout).fill_(float("nan"))


def assert_within(torch, got, want, bound, what):
    """|got - want| <= bound everywhere; want and bound are float64."""
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float(torch.nan_to_num(err / bound.clamp(min=1e-300)).max()))


# ---------------------------------------------------------------- layer norm

NORM_SIZES = [(1, 1), (1, 5), (3, 32), (5, 33), (2, 64), (130, 100), (7, 150), (9, 256), (4, 257), (33, 512), (6, 1000), (3, 1024),
              (3, 1027), (2, 2048), (5, 3001), (3, 4096), (2, 5000), (2, 8192), (2, 16384), (2100, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_layer_norm(gpu, ops, n, d, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    rng = np.random.default_rng(n * 7919 + d)
    for layout, affine in (("plain", True), ("odd", False), ("apart", True)):
        x = make_rows(torch, rng, n, d, t, layout)
        x += 3.0
        gamma = torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).float().to(DEV) if affine else None
        beta = torch.from_numpy(rng.standard_normal(d)).float().to(DEV) if affine else None
        y = empty_rows(torch, n, d, t, layout)
        mean, rstd = torch.full((n,), math.nan, device=DEV), torch.full((n,), math.nan, device=DEV)
        eps = 1e-3
        ops.sp_layer_norm(x, y, gamma=gamma, beta=beta, eps=eps, mean=mean, rstd=rstd)
        xd = x.double()
        m = xd.mean(1, keepdim=True)
        var = ((xd - m) ** 2).mean(1, keepdim=True)
        r = (var + eps).rsqrt()
        g = gamma.double() if affine else torch.ones(d, dtype=torch.float64, device=DEV)
        b = beta.double() if affine else torch.zeros(d, dtype=torch.float64, device=DEV)
        # the mean: a sum of d values in a tree no deeper than 64 in a lane and 16 across; 80 u of the mean magnitude
        dm = 84 * U * xd.abs().mean(1, keepdim=True)
        assert_within(torch, mean[:, None], m, dm, "mean")
        # the variance: the mean's error squared, and 84 u relative; rstd half of that and 4 u
        drel = 0.5 * (dm ** 2 + 84 * U * var) * r ** 2 + 6 * U
        assert_within(torch, rstd[:, None], r, drel * r, "rstd")
        xh = (xd - m) * r
        want = xh * g + b
        bound = ((dm + U * (xd - m).abs()) * r + xh.abs() * (drel + 2 * U)) * g.abs() + 3 * U * (xh * g).abs() + U * want.abs()
        bound = bound + half_step(torch, t) * (want.abs() + bound) + 1e-38
        assert_within(torch, y, want, bound, "y")


def test_layer_norm_of_equal_values_and_in_place(gpu, ops):
    torch, _ = gpu
    x = torch.full((5, 300), 7.25, device=DEV)          # sums of 7.25 are exact: a variance of exactly 0
    y = torch.empty_like(x)
    beta = torch.arange(300, device=DEV).float()
    ops.sp_layer_norm(x, y, beta=beta)
    assert torch.equal(y, beta.expand(5, 300))
    a = torch.randn(40, 300, device=DEV)
    want = torch.empty_like(a)
    ops.sp_layer_norm(a, want)
    ops.sp_layer_norm(a, a)
    assert torch.equal(a, want)


def norm_gradients(torch, dy, x, mean, rstd, gamma):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    g = gamma.double() if gamma is not None else torch.ones(x.shape[1], dtype=torch.float64, device=DEV)
    xh = (x - mean) * rstd
    q = dy * g
    dx = rstd * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
    size = rstd * (q.abs() + q.abs().mean(1, keepdim=True) + xh.abs() * (q * xh).abs().mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), size, (dy * xh).abs().sum(0), dy.abs().sum(0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_layer_norm_backward(gpu, ops, n, d, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    rng = np.random.default_rng(n * 104729 + d)
    for layout, affine in (("plain", True), ("odd", True), ("apart", False)):
        x = make_rows(torch, rng, n, d, t, layout)
        dy = make_rows(torch, rng, n, d, t, layout)
        gamma = torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).float().to(DEV) if affine else None
        mean = x.double().mean(1).float()
        rstd = (x.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
        dx = empty_rows(torch, n, d, t, layout)
        dgamma, dbeta = torch.full((d,), math.nan, device=DEV), torch.full((d,), math.nan, device=DEV)
        ops.sp_layer_norm_backward(dy, x, mean, rstd, gamma=gamma, dx=dx, dgamma=dgamma, dbeta=dbeta)
        wx, wg, wb, size, sg, sb = norm_gradients(torch, dy, x, mean, rstd, gamma)
        # xh: two roundings, the difference's error is relative to it (mean and rstd are inputs); sums over a row as above
        bound = 96 * U * size
        assert_within(torch, dx, wx, bound + half_step(torch, t) * (wx.abs() + bound) + 1e-38, "dx")
        assert_within(torch, dgamma, wg, (n + 8) * U * sg + 1e-38, "dgamma")
        assert_within(torch, dbeta, wb, (n + 8) * U * sb + 1e-38, "dbeta")
        again = [torch.empty_like(dgamma), torch.empty_like(dbeta)]
        ops.sp_layer_norm_backward(dy, x, mean, rstd, gamma=gamma, dgamma=again[0], dbeta=again[1])   # sums alone
        assert torch.equal(again[0], dgamma) and torch.equal(again[1], dbeta)


def test_layer_norm_gradient_against_differences(gpu, ops):
    """The directional derivative of sum(y c) in 64 bits, against the gradients' products with the direction."""
    torch, _ = gpu
    rng = np.random.default_rng(5)
    n, d, eps = 6, 70, 1e-5
    x, c, gamma, beta = (torch.from_numpy(rng.standard_normal(s)).float().to(DEV) for s in ((n, d), (n, d), (d,), (d,)))
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ops.sp_layer_norm(x, y, gamma=gamma, beta=beta, eps=eps, mean=mean, rstd=rstd)
    dx, dg, db = torch.empty_like(x), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    ops.sp_layer_norm_backward(c, x, mean, rstd, gamma=gamma, dx=dx, dgamma=dg, dbeta=db)

    def value(x_, g_, b_):
        m = x_.mean(1, keepdim=True)
        v = ((x_ - m) ** 2).mean(1, keepdim=True)
        return float((((x_ - m) / torch.sqrt(v + eps) * g_ + b_) * c.double()).sum())
    X, G, B = x.double(), gamma.double(), beta.double()
    for k in range(4):
        vx, vg, vb = (torch.from_numpy(rng.standard_normal(s)).to(DEV) for s in ((n, d), (d,), (d,)))
        h = 1e-4
        slope = (value(X + h * vx, G + h * vg, B + h * vb) - value(X - h * vx, G - h * vg, B - h * vb)) / (2 * h)
        parts = [(dx.double() * vx).sum(), (dg.double() * vg).sum(), (db.double() * vb).sum()]
        # float32 gradients: 1e-5 of the summed magnitudes covers their error; the differences' own is of order h^2
        size = float((dx.double() * vx).abs().sum() + (dg.double() * vg).abs().sum() + (db.double() * vb).abs().sum())
        assert abs(slope - float(sum(parts))) <= 1e-5 * size


def test_layer_norm_without_rows(gpu, ops):
    torch, _ = gpu
    x = torch.empty(0, 12, device=DEV)
    dg, db = torch.ones(12, device=DEV), torch.ones(12, device=DEV)
    e = torch.empty(0, device=DEV)
    ops.sp_layer_norm(x, x.clone(), mean=e, rstd=e.clone())
    ops.sp_layer_norm_backward(x, x.clone(), e, e.clone(), dgamma=dg, dbeta=db)
    assert not dg.any() and not db.any()


# ---------------------------------------------------------------- grouped linear layers

def offsets_of(torch, sizes):
    return torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device=DEV)


# rows of the groups, rows of no group, inputs, outputs
LINEAR_SIZES = [
    ((1,), 0, 1, 1), ((0, 1, 0), 0, 7, 3), ((0, 0), 3, 5, 4), ((5,), 0, 512, 256), ((1, 0, 2, 0, 0, 1), 2, 256, 1000), ((16,), 0, 64, 64),
    ((17, 15, 16), 0, 96, 33), ((3, 4), 0, 1500, 10), ((127,), 0, 32, 128), ((128,), 0, 40, 129), ((129, 1, 300), 5, 128, 64),
    ((257, 0, 64), 0, 150, 257), ((40, 41, 42, 43), 0, 31, 7), ((1000,), 3, 64, 130), ((700, 1, 900, 30), 0, 136, 200),
    ((1024, 2048), 0, 64, 96), ((200, 300), 11, 257, 65), ((3, 2) * 70, 4, 24, 20), ((5000,), 0, 16, 10), ((640, 385), 0, 256, 256),
]


def plain_linear(torch, x, sizes, w, bias, relu, residual):
    """Values and the bound's magnitudes, in 64 bits."""
    n, m = x.shape[0], w.shape[2]
    act = torch.zeros(n, m, dtype=torch.float64, device=DEV)
    size = torch.zeros_like(act)
    lo = 0
    for g, s in enumerate(sizes):
        rows = slice(lo, lo + s)
        lo += s
        act[rows] = x[rows].double() @ w[g].double()
        size[rows] = x[rows].double().abs() @ w[g].double().abs()
        if bias is not None:
            act[rows] += bias[g].double()
            size[rows] += bias[g].double().abs()
    if relu:
        act = act.clamp(min=0)
    y = act.clone()
    if residual is not None:
        y[:lo] += residual[:lo].double()
        size[:lo] += residual[:lo].double().abs()
    return y, act, size


@pytest.mark.parametrize("dtype", ["f32", "bf16", "bf16_to_f32"])
@pytest.mark.parametrize("sizes,spare,k,m", LINEAR_SIZES)
def test_grouped_linear(gpu, ops, sizes, spare, k, m, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype.split("_")[0])
    to = torch.float32 if dtype == "bf16_to_f32" else t
    n = sum(sizes) + spare
    rng = np.random.default_rng(n * 31 + k * 7 + m)
    offsets = offsets_of(torch, sizes)
    for layout, extras in (("plain", ()), ("odd", ("bias", "relu", "residual", "act")), ("apart", ("bias", "residual")),
                           ("plain", ("bias", "relu"))):
        x = make_rows(torch, rng, n, k, t, layout)
        if spare:
            x[n - spare:] = float("nan")                     # rows of no group touch nothing
        w = torch.from_numpy(rng.standard_normal((len(sizes), k, m)) / math.sqrt(k)).to(t).to(DEV)
        if layout == "odd":                                  # weights at an element's alignment, NaN around them
            store = torch.full((w.numel() + 2,), float("nan"), dtype=t, device=DEV)
            store[1:-1] = w.reshape(-1)
            w = store[1:-1].view(w.shape)
        bias = torch.from_numpy(rng.standard_normal((len(sizes), m))).float().to(DEV) if "bias" in extras else None
        residual = make_rows(torch, rng, n, m, to, layout) if "residual" in extras else None
        y = empty_rows(torch, n, m, to, layout)
        act = empty_rows(torch, n, m, to, layout) if "act" in extras else None
        ops.sp_grouped_linear(x, offsets, w, y, bias=bias, relu="relu" in extras, residual=residual, act_out=act)
        want, want_act, size = plain_linear(torch, x, sizes, w, bias, "relu" in extras, residual)
        bound = (k + 10) * U * size + 1e-36
        assert_within(torch, y, want, bound + half_step(torch, to) * (want.abs() + bound), "y")
        if act is not None:
            assert_within(torch, act, want_act, bound + half_step(torch, to) * (want_act.abs() + bound), "act_out")
        if residual is not None:                             # the sum may go where the residual was
            into = residual.clone() if layout == "plain" else residual
            ops.sp_grouped_linear(x, offsets, w, into, bias=bias, relu="relu" in extras, residual=into)
            assert torch.equal(into, y)


def plain_linear_backward(torch, dy, act, x, sizes, w):
    f64 = torch.float64
    dz = dy.double() if act is None else torch.where(act > 0, dy.double(), 0.0)
    n, k, groups, m = x.shape[0], x.shape[1], w.shape[0], w.shape[2]
    dx, sx = torch.zeros(n, k, dtype=f64, device=DEV), torch.zeros(n, k, dtype=f64, device=DEV)
    dw, sw = torch.zeros(groups, k, m, dtype=f64, device=DEV), torch.zeros(groups, k, m, dtype=f64, device=DEV)
    db, sb = torch.zeros(groups, m, dtype=f64, device=DEV), torch.zeros(groups, m, dtype=f64, device=DEV)
    lo = 0
    for g, s in enumerate(sizes):
        rows = slice(lo, lo + s)
        lo += s
        wt, xt = w[g].double().t().contiguous(), x[rows].double().t().contiguous()
        dx[rows], sx[rows] = dz[rows] @ wt, dz[rows].abs() @ wt.abs()
        dw[g], sw[g] = xt @ dz[rows], xt.abs() @ dz[rows].abs()
        db[g], sb[g] = dz[rows].sum(0), dz[rows].abs().sum(0)
    return dx, dw, db, sx, sw, sb


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,spare,k,m", LINEAR_SIZES)
def test_grouped_linear_backward(gpu, ops, sizes, spare, k, m, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    n = sum(sizes) + spare
    rng = np.random.default_rng(n * 37 + k * 11 + m)
    offsets = offsets_of(torch, sizes)
    longest = max(sizes)
    for layout, relu in (("plain", True), ("odd", True), ("apart", False), ("plain", False)):
        x, dy = make_rows(torch, rng, n, k, t, layout), make_rows(torch, rng, n, m, t, layout)
        act = make_rows(torch, rng, n, m, t, layout).clamp_(min=0) if relu else None
        if spare:
            x[n - spare:] = float("nan")
            dy[n - spare:] = float("nan")
        w = torch.from_numpy(rng.standard_normal((len(sizes), k, m)) / math.sqrt(k)).to(t).to(DEV)
        dx = empty_rows(torch, n, k, t, layout)
        dw = torch.full((len(sizes), k, m), math.nan, device=DEV)
        db = torch.full((len(sizes), m), math.nan, device=DEV)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, dx=dx, dw=dw, db=db)
        wx, ww, wb, sx, sw, sb = plain_linear_backward(torch, dy, act, x, sizes, w)
        bound = (m + 10) * U * sx + 1e-36
        assert_within(torch, dx, wx, bound + half_step(torch, t) * (wx.abs() + bound), "dx")
        assert_within(torch, dw, ww, (longest + 10) * U * sw + 1e-36, "dw")
        assert_within(torch, db, wb, (longest + 10) * U * sb + 1e-36, "db")
        # each gradient alone has the same bits
        one = empty_rows(torch, n, k, t, layout)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, dx=one)
        assert torch.equal(one, dx)
        one = torch.full_like(dw, math.nan)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, dw=one)
        assert torch.equal(one, dw)
        one = torch.full_like(db, math.nan)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, act=act, db=one)
        assert_within(torch, one, wb, (longest + 10) * U * sb + 1e-36, "db alone")


def test_linear_gradient_against_differences(gpu, ops):
    torch, _ = gpu
    rng = np.random.default_rng(8)
    sizes, k, m = (5, 0, 9), 12, 7
    n = sum(sizes)
    x, c = (torch.from_numpy(rng.standard_normal(s)).float().to(DEV) for s in ((n, k), (n, m)))
    w, b = (torch.from_numpy(rng.standard_normal(s)).float().to(DEV) for s in ((3, k, m), (3, m)))
    offsets = offsets_of(torch, sizes)
    y = torch.empty(n, m, device=DEV)
    ops.sp_grouped_linear(x, offsets, w, y, bias=b, relu=True)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ops.sp_grouped_linear_backward(c, x, offsets, w, act=y, dx=dx, dw=dw, db=db)

    def value(x_, w_, b_):
        return float((plain_linear(torch, x_, sizes, w_, b_, True, None)[0] * c.double()).sum())
    X, W, B = x.double(), w.double(), b.double()
    for _ in range(4):
        vx, vw, vb = (torch.from_numpy(rng.standard_normal(tuple(s.shape))).to(DEV) for s in (x, w, b))
        h = 1e-6                                            # no unit of this draw changes sign within it
        slope = (value(X + h * vx, W + h * vw, B + h * vb) - value(X - h * vx, W - h * vw, B - h * vb)) / (2 * h)
        parts = [(dx.double() * vx), (dw.double() * vw), (db.double() * vb)]
        assert abs(slope - float(sum(p.sum() for p in parts))) <= 1e-5 * float(sum(p.abs().sum() for p in parts))


def test_linear_nan_and_infinity_stay_in_their_rows(gpu, ops):
    torch, _ = gpu
    for t in (torch.float32, torch.bfloat16):
        sizes, k, m = (70, 60), 100, 90
        x = torch.randn(130, k, device=DEV).to(t)
        w = torch.randn(2, k, m, device=DEV).to(t)
        offsets = offsets_of(torch, sizes)
        want = torch.empty(130, m, dtype=t, device=DEV)
        ops.sp_grouped_linear(x, offsets, w, want, relu=True)
        x[69, 99], x[3, 0] = math.nan, math.inf
        y = torch.empty_like(want)
        ops.sp_grouped_linear(x, offsets, w, y, relu=True)
        assert bool(y[69].isnan().all())
        assert not bool(y[3].isfinite().logical_and(y[3] > 0).any())
        keep = [i for i in range(130) if i not in (3, 69)]
        assert torch.equal(y[keep], want[keep])
        dy = torch.randn(130, m, device=DEV).to(t)
        dw, db = torch.empty(2, k, m, device=DEV), torch.empty(2, m, device=DEV)
        dw0, db0 = torch.empty_like(dw), torch.empty_like(db)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, dw=dw, db=db)
        x[69, 99] = x[3, 0] = 0
        ops.sp_grouped_linear_backward(dy, x, offsets, w, dw=dw0, db=db0)
        assert torch.equal(dw[1], dw0[1]) and torch.equal(db, db0)      # the other group has not seen them
        assert bool(dw[0, 99].isnan().all()) and torch.equal(dw[0, 1:99], dw0[0, 1:99])


@pytest.mark.parametrize("bad", [(1, 4, 8), (0, 9, 8), (0, 4, 99), (0, -3, 8), (0, 4, -1)])
def test_bad_offsets_are_reported_and_followed_nowhere(gpu, ops, bad):
    torch, binding = gpu
    n, k, m = 8, 6, 5
    x, w = torch.randn(n, k, device=DEV), torch.randn(2, k, m, device=DEV)
    guard = torch.full((3 * n, m), 7.0, device=DEV)
    offsets = torch.tensor(bad, dtype=torch.int32, device=DEV)
    ops.sp_grouped_linear(x, offsets, w, guard[n:2 * n])
    with pytest.raises(binding.SneakPeekError) as e:
        ops.sp_ops_check()
    assert e.value.status == binding.SP_EINVAL
    ops.sp_ops_check()                                        # reported once
    assert bool((guard[:n] == 7).all()) and bool((guard[2 * n:] == 7).all())
    dw = torch.empty_like(w)
    ops.sp_grouped_linear_backward(guard[n:2 * n], x, offsets, w, dw=dw)
    with pytest.raises(binding.SneakPeekError):
        ops.sp_ops_check()


# ---------------------------------------------------------------- loss

def plain_loss(torch, z, classes, label, weight, scale):
    """Losses, gradients and the bounds' magnitudes in 64 bits; classes per row."""
    zd = z.double()
    n, c_max = z.shape
    inside = torch.arange(c_max, device=DEV)[None] < classes[:, None]
    zd = torch.where(inside, zd, -math.inf)
    top = zd.max(1, keepdim=True).values
    none = (label < 0) | (top[:, 0] == -math.inf)
    top = torch.where(none[:, None], 0.0, top)
    e = torch.exp(zd - top)
    total = torch.where(none, 1.0, e.sum(1))[:, None]
    w = torch.where(none, 0.0, torch.ones_like(total[:, 0]) if weight is None else weight.double())
    at = label.clamp(min=0).long()[:, None]
    zl = torch.where(none, 0.0, zd.gather(1, at)[:, 0])
    loss = torch.where(none, 0.0, (torch.log(total[:, 0]) + top[:, 0] - zl) * w)
    p = torch.where(none[:, None], 0.0, e / total)
    hit = (torch.arange(c_max, device=DEV)[None] == at).double()
    grad = torch.where(none[:, None], 0.0, (p - hit) * (w * scale)[:, None])
    return loss, grad, p, (torch.log(total[:, 0]).abs() + top[:, 0].abs() + zl.abs()) * w, (p + hit) * (w * abs(scale))[:, None]


LOSS_SIZES = [(1, 1), (1, 2), (5, 10), (70, 31), (33, 33), (20, 64), (9, 100), (40, 257), (10, 1000), (3, 1024), (5, 1030), (4, 2048),
              (3, 4097), (2, 9000), (3, 16384), (2, 16390), (2, 40001), (9000, 7)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f32_to_bf16"])
@pytest.mark.parametrize("n,c_max", LOSS_SIZES)
def test_cross_entropy(gpu, ops, n, c_max, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype.split("_")[0])
    tg = torch.bfloat16 if dtype == "f32_to_bf16" else t
    rng = np.random.default_rng(n * 13 + c_max)
    for layout, ragged, weighted in (("plain", False, False), ("odd", True, True), ("apart", True, False)):
        apps = 5
        z = make_rows(torch, rng, n, c_max, t, layout, scale=4.0)
        n_classes = torch.from_numpy(rng.integers(1, c_max + 1, apps)).int().to(DEV)
        app = torch.from_numpy(rng.integers(0, apps, n)).int().to(DEV) if ragged else None
        classes = n_classes[app.long()] if ragged else torch.full((n,), c_max, dtype=torch.int32, device=DEV)
        label = (torch.from_numpy(rng.random(n)).to(DEV) * classes).int().clamp(max=c_max - 1)
        label[torch.from_numpy(rng.random(n) < 0.2).to(DEV)] = -1
        if ragged:                                            # what lies beyond the classes is not read
            z[torch.arange(c_max, device=DEV)[None] >= classes[:, None]] = math.nan
        weight = torch.from_numpy(rng.random(n)).float().to(DEV) if weighted else None
        loss = torch.full((n,), math.nan, device=DEV)
        dz = empty_rows(torch, n, c_max, tg, layout)
        scale = 0.37
        ops.sp_cross_entropy(z, label, loss, app=app, n_classes=n_classes if ragged else None, weight=weight, scale=scale, dlogits=dz)
        want, grad, p, size, gsize = plain_loss(torch, z, classes, label, weight, scale)
        # exp of a difference d is off by (1 + |d|) u for the difference's rounding and 2 u of its own; differences reach 60 here only
        # where exp has nothing left; sums as above; the logarithm adds the relative error of the sum
        rel = 64 * U
        assert_within(torch, loss, want, rel * (torch.ones_like(want) + size) + 1e-38, "loss")
        bound = 2 * rel * gsize + 1e-38
        assert_within(torch, dz, grad, bound + half_step(torch, tg) * (grad.abs() + bound), "dlogits")
        alone = torch.empty_like(loss)
        ops.sp_cross_entropy(z, label, alone, app=app, n_classes=n_classes if ragged else None, weight=weight, scale=scale)
        assert torch.equal(alone, loss)
        if tg == t:                                           # gradients may take the logits' place
            ops.sp_cross_entropy(z, label, alone, app=app, n_classes=n_classes if ragged else None, weight=weight, scale=scale, dlogits=z)
            assert torch.equal(alone, loss) and torch.equal(z, dz)


@pytest.mark.parametrize("c", [6, 300, 3000, 20000])
def test_cross_entropy_masks(gpu, ops, c):
    """Logits of the type's lowest value and of -inf, rows in which nothing is left, infinities and NaN."""
    torch, _ = gpu
    for t in (torch.float32, torch.bfloat16):
        lowest = torch.finfo(t).min
        z = torch.randn(8, c, device=DEV).to(t)
        z[0, 1:] = -math.inf                                  # one class left, and it is the label
        z[1, :] = -math.inf                                   # none left
        z[2, :] = lowest                                      # all masked by the lowest value: even odds
        z[3, 2:] = lowest
        z[4, 0] = -math.inf                                   # the label cannot be
        z[5, c - 1] = math.nan
        z[6, 0] = math.inf
        z[7, :] = math.nan
        label = torch.tensor([0, 0, 1, 1, 0, 0, 0, 0], dtype=torch.int32, device=DEV)
        loss = torch.empty(8, device=DEV)
        dz = torch.empty_like(z)
        ops.sp_cross_entropy(z, label, loss, dlogits=dz)
        assert float(loss[0]) == 0 and not dz[0].any()
        assert float(loss[1]) == 0 and not dz[1].any()
        assert abs(float(loss[2]) - math.log(c)) <= 64 * U * (1 + math.log(c))
        e = half_step(torch, t) + 64 * U
        assert abs(float(dz[2, 0]) - 1 / c) <= e / c and abs(float(dz[2, 1]) - (1 / c - 1)) <= e
        assert not dz[3, 2:].any() and abs(float(dz[3, 0]) + float(dz[3, 1])) <= 2 * e
        assert float(loss[4]) == math.inf and float(dz[4, 0]) == -1.0
        for row in (5, 6, 7):
            assert math.isnan(float(loss[row])) and bool(dz[row].isnan().any())


def test_cross_entropy_gradient_against_differences(gpu, ops):
    torch, _ = gpu
    rng = np.random.default_rng(3)
    n, c = 12, 9
    z = torch.from_numpy(rng.standard_normal((n, c))).float().to(DEV)
    label = torch.from_numpy(rng.integers(0, c, n)).int().to(DEV)
    weight = torch.from_numpy(rng.random(n)).float().to(DEV)
    loss, dz = torch.empty(n, device=DEV), torch.empty_like(z)
    ops.sp_cross_entropy(z, label, loss, weight=weight, scale=0.25, dlogits=dz)
    classes = torch.full((n,), c, device=DEV)
    value = lambda q: 0.25 * float(plain_loss(torch, q, classes, label, weight, 1.0)[0].sum())
    Z = z.double()
    for _ in range(4):
        v = torch.from_numpy(rng.standard_normal((n, c))).to(DEV)
        h = 1e-4
        slope = (value(Z + h * v) - value(Z - h * v)) / (2 * h)
        assert abs(slope - float((dz.double() * v).sum())) <= 1e-5 * float((dz.double() * v).abs().sum())


def test_cross_entropy_reports_bad_rows(gpu, ops):
    torch, binding = gpu
    z = torch.randn(4, 5, device=DEV)
    n_classes = torch.tensor([5, 3, 0, 6], dtype=torch.int32, device=DEV)
    good = dict(app=[0, 1, 0, 1], label=[4, 2, -1, 0])
    for change in (dict(app=[0, 4, 0, 1]), dict(app=[0, -1, 0, 1]), dict(app=[0, 2, 0, 1]), dict(app=[0, 3, 0, 1]),
                   dict(label=[4, 3, -1, 0]), dict(label=[4, -2, -1, 0])):
        case = {**good, **change}
        app, label = (torch.tensor(case[k], dtype=torch.int32, device=DEV) for k in ("app", "label"))
        loss, dz = torch.full((4,), 9.0, device=DEV), torch.full((4, 5), 9.0, device=DEV)
        ops.sp_cross_entropy(z, label, loss, app=app, n_classes=n_classes, dlogits=dz)
        with pytest.raises(binding.SneakPeekError) as e:
            ops.sp_ops_check()
        assert e.value.status == binding.SP_EINVAL
        assert float(loss[1]) == 0 and not dz[1].any() and float(loss[0]) > 0
    ops.sp_cross_entropy(z, torch.tensor(good["label"], dtype=torch.int32, device=DEV), torch.empty(4, device=DEV),
                         app=torch.tensor(good["app"], dtype=torch.int32, device=DEV), n_classes=n_classes)
    ops.sp_ops_check()


# ---------------------------------------------------------------- clipping

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [(1,), (0, 3, 0), (5, 17, 1000), (16384, 16385, 40000), (7,) * 300, (100003,), (250000, 1, 250001)])
def test_clip_grad_norm(gpu, ops, sizes, dtype):
    torch, binding = gpu
    t = dtype_of(torch, dtype)
    rng = np.random.default_rng(sum(sizes))
    flat = torch.from_numpy(rng.standard_normal(sum(sizes))).to(t).to(DEV)
    grads = list(flat.split(list(sizes)))                     # views at every alignment
    norm = torch.full((1,), math.nan, device=DEV)
    exact = math.sqrt(float((flat.double() ** 2).sum()))
    for limit in (0.5, 1e9, 0.0):
        out = torch.full_like(flat, math.nan)
        ops.sp_clip_grad_norm(binding.TensorList(grads, out=out.split(list(sizes))), limit, norm)
        assert abs(float(norm) - exact) <= 2 * U * exact
        c = min(1.0, limit / (exact + 1e-6))
        want = flat.double() * c
        assert_within(torch, out, want, (3 * U + half_step(torch, t)) * want.abs() + 1e-40, "clipped")
        if limit > exact:
            assert torch.equal(out, flat)                     # nothing to scale: nothing changes
    before = flat.clone()
    ops.sp_clip_grad_norm(grads, 0.5, norm)                   # in place
    c = min(1.0, 0.5 / (exact + 1e-6))
    want = before.double() * c
    assert_within(torch, flat, want, (3 * U + half_step(torch, t)) * want.abs() + 1e-40, "in place")


def test_clip_extremes(gpu, ops):
    torch, binding = gpu
    norm = torch.full((1,), 5.0, device=DEV)
    ops.sp_clip_grad_norm([], 1.0, norm)
    assert float(norm) == 0
    zeros = torch.zeros(1000, device=DEV)
    ops.sp_clip_grad_norm([zeros], 1.0, norm)
    assert float(norm) == 0 and not zeros.any()
    huge = torch.full((4,), 1e30, device=DEV)                 # squares beyond float32's range
    ops.sp_clip_grad_norm([huge], 1.0, norm)
    assert abs(float(norm) / 2e30 - 1) <= 2 * U and abs(float(huge[0]) - 0.5) <= 4 * U
    tiny = torch.full((4,), 1e-30, device=DEV)
    ops.sp_clip_grad_norm([tiny], 1.0, norm)
    assert abs(float(norm) / 2e-30 - 1) <= 2 * U
    inf = torch.tensor([1.0, math.inf], device=DEV)
    ops.sp_clip_grad_norm([inf], 1.0, norm)
    assert float(norm) == math.inf and float(inf[0]) == 0 and math.isnan(float(inf[1]))
    nan = torch.tensor([1.0, math.nan], device=DEV)
    ops.sp_clip_grad_norm([nan], 1.0, norm)
    assert math.isnan(float(norm)) and bool(nan.isnan().all())
    ops.sp_clip_grad_norm([torch.ones(4, device=DEV)], 1.0, norm)
    assert float(norm) == 2


# ---------------------------------------------------------------- all of them

def head_step(torch, ops, t, state, stream=None):
    """Layer norm, hidden layer, logits, loss and all gradients of three applications' heads, clipped."""
    s = state
    ops.sp_layer_norm(s["x"], s["xn"], gamma=s["gamma"], beta=s["beta"], mean=s["mean"], rstd=s["rstd"], stream=stream)
    ops.sp_grouped_linear(s["xn"], s["offsets"], s["w1"], s["h"], bias=s["b1"], relu=True, stream=stream)
    ops.sp_grouped_linear(s["h"], s["offsets"], s["w2"], s["z"], bias=s["b2"], stream=stream)
    ops.sp_cross_entropy(s["z"], s["label"], s["loss"], app=s["app"], n_classes=s["n_classes"], scale=0.01, dlogits=s["dz"], stream=stream)
    ops.sp_grouped_linear_backward(s["dz"], s["h"], s["offsets"], s["w2"], dx=s["dh"], dw=s["dw2"], db=s["db2"], stream=stream)
    ops.sp_grouped_linear_backward(s["dh"], s["xn"], s["offsets"], s["w1"], act=s["h"], dx=s["dxn"], dw=s["dw1"], db=s["db1"], stream=stream)
    ops.sp_layer_norm_backward(s["dxn"], s["x"], s["mean"], s["rstd"], gamma=s["gamma"], dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"],
                               stream=stream)
    ops.sp_clip_grad_norm(s["list"], 0.01, s["norm"], stream=stream)


def head_state(torch, binding, t, sizes, d, h, c, seed):
    rng = np.random.default_rng(seed)
    n, a = sum(sizes), len(sizes)
    f = lambda *s, scale=1.0, dt=torch.float32: (torch.from_numpy(rng.standard_normal(s)) * scale).to(dt).to(DEV)
    e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=DEV)
    s = dict(x=f(n, d, dt=t), gamma=1 + f(d, scale=0.1), beta=f(d, scale=0.1), w1=f(a, d, h, scale=d ** -0.5, dt=t), b1=f(a, h),
             w2=f(a, h, c, scale=h ** -0.5, dt=t), b2=f(a, c), offsets=offsets_of(torch, sizes),
             app=torch.repeat_interleave(torch.arange(a, dtype=torch.int32), torch.tensor(sizes)).to(DEV),
             n_classes=torch.tensor([c - i for i in range(a)], dtype=torch.int32, device=DEV),
             label=torch.from_numpy(rng.integers(-1, c - a, n)).int().to(DEV),
             xn=e(n, d, dt=t), mean=e(n), rstd=e(n), h=e(n, h, dt=t), z=e(n, c), loss=e(n), dz=e(n, c, dt=t), dh=e(n, h, dt=t),
             dw2=e(a, h, c), db2=e(a, c), dw1=e(a, d, h), db1=e(a, h), dxn=e(n, d, dt=t), dx=e(n, d, dt=t), dgamma=e(d), dbeta=e(d), norm=e(1))
    s["list"] = binding.TensorList([s[k] for k in ("dw1", "db1", "dw2", "db2", "dgamma", "dbeta")])
    return s


OUTPUTS = ("xn", "mean", "rstd", "h", "z", "loss", "dz", "dh", "dw2", "db2", "dw1", "db1", "dxn", "dx", "dgamma", "dbeta", "norm")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_repeats_bit_for_bit_on_any_stream_and_in_a_graph(gpu, ops, dtype):
    torch, binding = gpu
    t = dtype_of(torch, dtype)
    s = head_state(torch, binding, t, (1500, 0, 700), 128, 64, 10, 4)
    head_step(torch, ops, t, s)
    torch.cuda.synchronize()
    want = {k: s[k].clone() for k in OUTPUTS}

    def wipe():
        for k in OUTPUTS:
            s[k].fill_(math.nan)

    wipe()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    head_step(torch, ops, t, s, stream=side)
    side.synchronize()
    for k in OUTPUTS:
        assert torch.equal(s[k], want[k]), k

    wipe()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        head_step(torch, ops, t, s)
    for _ in range(4):
        wipe()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in OUTPUTS:
            assert torch.equal(s[k], want[k]), k
        other = head_state(torch, binding, t, (300, 11), 64, 32, 5, 9)
        head_step(torch, ops, t, other)                       # the program's own work between replays
    ops.sp_ops_check()


def test_a_small_workspace_gives_the_same_results(gpu, ops):
    torch, binding = gpu
    small = binding.Ops(workspace_bytes=1 << 20)
    for t in (torch.float32, torch.bfloat16):
        s = head_state(torch, binding, t, (9000, 0, 3000), 256, 64, 12, 6)
        head_step(torch, small, t, s)
        wx, ww, wb, sx, sw, sb = plain_linear_backward(torch, s["dh"], s["h"], s["xn"], (9000, 0, 3000), s["w1"])
        c = min(1.0, 0.01 / (float(s["norm"]) + 1e-6))
        assert_within(torch, s["dw1"], ww * c, (9010 + 4) * U * sw * c + 1e-36, "dw")
        assert_within(torch, s["db1"], wb * c, (9010 + 4) * U * sb * c + 1e-36, "db")
        _, wg, wbt, _, sg, sbt = norm_gradients(torch, s["dxn"], s["x"], s["mean"], s["rstd"], s["gamma"])
        assert_within(torch, s["dgamma"], wg * c, 12020 * U * sg * c + 1e-36, "dgamma")
    small.sp_ops_check()
    small.close()


def test_rows_beyond_32_bit_offsets(gpu, ops):
    """Rows whose elements lie more than 2^31 elements into their array."""
    torch, _ = gpu
    n, d = 2_200_000, 1024                                    # 2.25e9 elements
    x = torch.zeros(n, d, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(5, d, device=DEV).to(torch.bfloat16)
    x[-5:] = tail
    y = torch.empty_like(x)
    ops.sp_layer_norm(x, y)
    small = torch.empty_like(tail)
    ops.sp_layer_norm(tail, small)
    assert torch.equal(y[-5:], small)
    label = torch.zeros(n, dtype=torch.int32, device=DEV)
    loss, few = torch.empty(n, device=DEV), torch.empty(5, device=DEV)
    ops.sp_cross_entropy(x, label, loss, dlogits=y)
    ops.sp_cross_entropy(tail, label[:5], few, dlogits=small)
    assert torch.equal(loss[-5:], few) and torch.equal(y[-5:], small)
    offsets = torch.tensor([0, n - 5, n], dtype=torch.int32, device=DEV)
    w = torch.randn(2, d, 8, device=DEV).to(torch.bfloat16)
    out = torch.empty(n, 8, dtype=torch.bfloat16, device=DEV)
    ops.sp_grouped_linear(x, offsets, w, out)
    want = tail.double() @ w[1].double()
    size = tail.double().abs() @ w[1].double().abs()
    bound = (d + 10) * U * size
    assert_within(torch, out[-5:], want, bound + half_step(torch, torch.bfloat16) * (want.abs() + bound), "y")
    dw = torch.empty(2, d, 8, device=DEV)
    dx = y
    ops.sp_grouped_linear_backward(out, x, offsets, w, dx=dx, dw=dw)
    want = tail.double().t().contiguous() @ out[-5:].double()
    assert_within(torch, dw[1], want, 15 * U * (tail.double().abs().t().contiguous() @ out[-5:].double().abs()), "dw")
    assert not dw[0].any()
    want = out[-5:].double() @ w[1].double().t().contiguous()
    bound = 18 * U * (out[-5:].double().abs() @ w[1].double().abs().t().contiguous())
    assert_within(torch, dx[-5:], want, bound + half_step(torch, torch.bfloat16) * (want.abs() + bound), "dx")


def test_what_does_not_fit_together_is_refused(gpu, ops):
    torch, binding = gpu
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=DEV)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    x, off, w, y = z(4, 8), i(3), z(2, 8, 6), z(4, 6)
    refused = [
        lambda: ops.sp_layer_norm(x, z(4, 7)), lambda: ops.sp_layer_norm(x, z(4, 8, dt=torch.bfloat16)), lambda: ops.sp_layer_norm(x.half(), x.half()),
        lambda: ops.sp_layer_norm(x.t(), z(8, 4)), lambda: ops.sp_layer_norm(x, z(4, 8), gamma=z(7)), lambda: ops.sp_layer_norm(x.cpu(), z(4, 8)),
        lambda: ops.sp_layer_norm(x, z(4, 8), mean=z(5)), lambda: ops.sp_layer_norm(x[:1].expand(4, 8), z(4, 8)),
        lambda: ops.sp_layer_norm_backward(z(4, 7), x, z(4), z(4), dx=z(4, 8)), lambda: ops.sp_layer_norm_backward(x, x, z(4), z(4), dgamma=z(9)),
        lambda: ops.sp_grouped_linear(x, off, z(2, 7, 6), y), lambda: ops.sp_grouped_linear(x, i(2), w, y), lambda: ops.sp_grouped_linear(x, off.long(), w, y),
        lambda: ops.sp_grouped_linear(x, off, w.transpose(1, 2), z(4, 8)), lambda: ops.sp_grouped_linear(x, off, w, z(5, 6)),
        lambda: ops.sp_grouped_linear(x, off, w, z(4, 6, dt=torch.bfloat16)), lambda: ops.sp_grouped_linear(x, off, w, y, bias=z(6)),
        lambda: ops.sp_grouped_linear(x, off, w, y, residual=z(4, 6, dt=torch.bfloat16)), lambda: ops.sp_grouped_linear(x, off, w.bfloat16(), y),
        lambda: ops.sp_grouped_linear_backward(y, x, off, w, dw=z(2, 6, 8)), lambda: ops.sp_grouped_linear_backward(z(4, 8), x, off, w, dx=x),
        lambda: ops.sp_grouped_linear_backward(y, x, off, w, act=z(4, 5), dx=z(4, 8)),
        lambda: ops.sp_cross_entropy(y, i(5), z(4)), lambda: ops.sp_cross_entropy(y, i(4).long(), z(4)), lambda: ops.sp_cross_entropy(y, i(4), z(4), app=i(4)),
        lambda: ops.sp_cross_entropy(y, i(4), z(4), dlogits=z(4, 5)), lambda: ops.sp_cross_entropy(y.bfloat16(), i(4), z(4), dlogits=z(4, 6)),
        lambda: ops.sp_clip_grad_norm([x.t()], 1.0, z(1)), lambda: ops.sp_clip_grad_norm([x, x.bfloat16()], 1.0, z(1)),
        lambda: ops.sp_clip_grad_norm([x], 1.0, z(2)), lambda: ops.sp_clip_grad_norm([x], 1.0, z(1), out=[y]), lambda: ops.sp_clip_grad_norm([x.cpu()], 1.0, z(1)),
        lambda: ops.sp_clip_grad_norm([x], -1.0, z(1)),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(binding.SneakPeekError) as e:
            call()
        assert e.value.status == binding.SP_EINVAL, k


@pytest.mark.parametrize("args", [[], ["--bf16"]])
def test_the_example_learns_and_serves(gpu, args):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_heads.py")
    spec = importlib.util.spec_from_file_location("train_heads", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    losses, trained, seen, summary = module.main(args + ["--steps", "120"])
    assert losses[-1] < 0.5 * losses[0] and trained > 0.8 and seen > 0.7
    assert summary["done"] == 1 and summary["n_scheduled"] > 0
