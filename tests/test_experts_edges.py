"""The ends of the ranges of the operators for heads that are made of experts, on the GPU, against their definitions in 64 bits: numbers far from one,
and so many rows that a launch's workgroups, or teams in them, take several in turn."""
import math

import numpy as np
import pytest

from tests.test_experts import (DEV, INF, U, assert_within, dtype_of, gpu, half_step, in_layout, ops, philox,  # noqa: F401 (fixtures)
                                quantized_layer, run_route, weights_by_definition)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- 8 bits

@pytest.mark.parametrize("n,k,m,groups", [(6, 96, 70, 2), (300, 33, 20, 3), (40000, 64, 64, 3), (33000, 65, 70, 2), (40001, 128, 200, 2), (131100, 1040, 1030, 3)])
def test_grouped_linear_quantized_of_rows_far_from_one(gpu, ops, n, k, m, groups):
    """The sum times a row's scale may pass float32 where the result does not; rows of ordinary size lie next to such rows."""
    torch, _ = gpu
    rng = np.random.default_rng(n + k)
    x = torch.from_numpy(rng.integers(-127, 128, (n, k)).astype(np.int8)).to(DEV)
    w = torch.from_numpy(rng.integers(-127, 128, (groups, m, k)).astype(np.int8)).to(DEV)
    # scales of rows up to that of float32's largest number, and of outputs that bring the largest sums, 127 * 127 * 1040 < 2^25, back below 2^128
    up = torch.from_numpy(rng.choice([-100, -10, 0, 30, 63, 64, 65, 100, 120], n)).to(DEV)
    down = torch.from_numpy(rng.choice([-120, -100, -70, -40], (groups, m))).to(DEV)
    up[:: 7] = 0                                           # (some tiles hold both kinds)
    up[n // 2:n // 2 + min(300, n // 3)] = 0               # (and some the ordinary one only)
    xs = (torch.from_numpy(rng.random(n) + 0.5).to(DEV) * torch.exp2(up.double())).float()
    ws = (torch.from_numpy(rng.random((groups, m)) + 0.5).to(DEV) * torch.exp2(down.double())).float()
    cuts = np.sort(rng.integers(0, n + 1, groups - 1))
    offsets = torch.from_numpy(np.concatenate([[0], cuts, [n]]).astype(np.int32)).to(DEV)
    for with_more in (False, True):
        bias = torch.from_numpy(rng.standard_normal((groups, m))).float().to(DEV) if with_more else None
        r = torch.from_numpy(rng.standard_normal((n, m))).float().to(DEV) if with_more else None
        y = torch.full((n, m), math.nan, device=DEV)
        ops.sp_grouped_linear_quantized(x, xs, offsets, w, ws, y, bias=bias, relu=with_more, residual=r)
        want, bound = quantized_layer(torch, x, xs, offsets, w, ws, bias, with_more, r)
        fits = want.abs() < 2.0 ** 127
        assert float(fits.double().mean()) > 0.9
        assert_within(torch, torch.where(fits, y, 0.0), torch.where(fits, want, 0.0), bound + U * (want.abs() + bound), ("y", with_more))
    ops.sp_ops_check()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,k,m", [(40, 64, 70), (2100, 1024, 1000), (2100, 1019, 1000)])
def test_grouped_linear_quantized_of_rows_as_far_apart_as_may_be(gpu, ops, n, k, m):
    torch, _ = gpu
    far = 8388608                                          # SP_MAX_LINEAR_STRIDE; 128 rows of it pass 2^30 bytes, all of them 2^32
    g = torch.Generator(device=DEV).manual_seed(n + k)
    x = torch.zeros((n - 1) * far + k, dtype=torch.int8, device=DEV).as_strided((n, k), (far, 1))
    x.copy_(torch.randint(-127, 128, (n, k), dtype=torch.int8, device=DEV, generator=g))
    w = torch.randint(-127, 128, (2, m, k), dtype=torch.int8, device=DEV, generator=g)
    xs, ws = torch.rand(n, device=DEV, generator=g) + 0.01, torch.rand(2, m, device=DEV, generator=g) + 0.01
    offsets = torch.tensor([0, n // 3, n], dtype=torch.int32, device=DEV)
    y = torch.full((n, m), math.nan, device=DEV)
    ops.sp_grouped_linear_quantized(x, xs, offsets, w, ws, y)
    want, bound = quantized_layer(torch, x.contiguous(), xs, offsets, w, ws, None, False, None)
    assert_within(torch, y, want, bound + U * (want.abs() + bound), "y")
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [33, 3000])
def test_grouped_linear_quantized_of_weights_beyond_32_bits(gpu, ops, n):
    torch, _ = gpu
    groups, m, k = 66, 8192, 8192                          # 4.4e9 weights
    g = torch.Generator(device=DEV).manual_seed(n)
    w = torch.randint(-127, 128, (groups, m, k), dtype=torch.int8, device=DEV, generator=g)
    x = torch.randint(-127, 128, (n, k), dtype=torch.int8, device=DEV, generator=g)
    xs, ws = torch.rand(n, device=DEV, generator=g) + 0.01, torch.rand(groups, m, device=DEV, generator=g) + 0.01
    ends = torch.zeros(groups + 1, dtype=torch.int32, device=DEV)
    ends[32:], ends[64:], ends[65:], ends[66] = n // 4, n // 3, n // 2, n
    y = torch.full((n, m), math.nan, device=DEV)
    ops.sp_grouped_linear_quantized(x, xs, ends, w, ws, y)
    want, bound = quantized_layer(torch, x, xs, ends, w, ws, None, False, None)
    assert_within(torch, y, want, bound + U * (want.abs() + bound), "y")
    del w
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- many rows

def routed(torch, z, top, sigmoid, bias, groups, top_groups):
    """Chosen experts in 64 bits, all rows at once.  z float64 with -inf for experts that are not there."""
    n, experts = z.shape
    there = z > -INF
    if bias is None and groups == 1:
        c = z
    else:
        c = torch.sigmoid(z) if sigmoid else torch.softmax(torch.where(there, z, -1e6), 1)
        if bias is not None:
            c = c + bias.double()
    c = torch.where(there, c, -INF)
    if groups > 1:
        by = c.view(n, groups, experts // groups)
        best = by.sort(dim=2, descending=True).values[:, :, :2]
        value = torch.where(best[:, :, 0] > -INF, torch.where(best > -INF, best, 0.0).sum(2), -INF)
        keep = value.sort(dim=1, descending=True, stable=True).indices[:, :top_groups]
        stays = torch.zeros_like(value, dtype=torch.bool).scatter(1, keep, True)
        c = torch.where(stays[:, :, None], by, -INF).reshape(n, experts)
    value, at = c.sort(dim=1, descending=True, stable=True)
    return torch.where(value[:, :top] > -INF, at[:, :top], -1)


# 65536 rows at once in teams of 8, 8192 in wavefronts (more than 8 chosen); 56 and 63 rows that are put off before they are taken
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,experts,top,groups,top_groups", [(70001, 256, 8, 8, 4), (600001, 16, 8, 1, 1), (600001, 24, 6, 4, 3), (9001, 300, 8, 1, 1),
                                                             (560001, 24, 9, 1, 1), (560001, 24, 9, 3, 2)])
def test_route_of_many_rows(gpu, ops, n, experts, top, groups, top_groups, dtype):
    torch, _ = gpu
    g = torch.Generator(device=DEV).manual_seed(n + experts)
    t = dtype_of(torch, dtype)
    for sigmoid, biased, renormalize in ((False, False, True), (True, True, True), (False, True, False)):
        z = torch.randn(n, experts, device=DEV, generator=g) * 1.5
        # most rows of the second third have too few experts; some rows none, some of the last third all of them alike
        z[n // 3:2 * n // 3].masked_fill_(torch.rand(2 * n // 3 - n // 3, experts, device=DEV, generator=g) < 0.75, -INF)
        z[:: 97] = -INF
        z[2 * n // 3:][:: 3] = 0.5
        z = z.to(t)
        bias = (torch.randn(experts, device=DEV, generator=g) * 0.1) if biased else None
        kw = dict(sigmoid=sigmoid, renormalize=renormalize, scale=2.5)
        expert, weight = run_route(torch, ops, z, top, bias=bias, groups=groups, top_groups=top_groups, **kw)
        want = routed(torch, z.double(), top, sigmoid, bias, groups, top_groups)
        assert torch.equal(expert.long(), want), int((expert.long() != want).any(1).sum())
        w, bound = weights_by_definition(torch, z.double(), want, sigmoid, renormalize, 2.5)
        some = (want >= 0).any(1)                          # (a row without an expert has weights of 0; its bound is a quotient of zeros)
        assert_within(torch, weight[some], w[some], bound[some], "weight")
        assert bool((weight[~some] == 0).all())
    ops.sp_ops_check()


# 32768 rows of more than 32 pieces of 16 bytes at once, 262144 of up to 8
@pytest.mark.parametrize("n,experts,top,dtype", [(40001, 256, 8, "f32"), (40001, 1000, 20, "bf16"), (70001, 100, 4, "f32"), (270001, 16, 4, "bf16"), (270001, 30, 3, "f32")])
def test_route_backward_of_many_rows(gpu, ops, n, experts, top, dtype):
    torch, _ = gpu
    g = torch.Generator(device=DEV).manual_seed(n + experts)
    t = dtype_of(torch, dtype)
    z = (torch.randn(n, experts, device=DEV, generator=g) * 2).to(t)
    z.masked_fill_(torch.rand(n, experts, device=DEV, generator=g) < 0.1, -INF)
    z[:: 101] = -INF
    zd = z.double()
    expert = routed(torch, zd, top, False, None, 1, 1).int()
    expert[5:: 7, 0] = -1                                  # dropped afterwards
    dw = torch.randn(n, top, device=DEV, generator=g)
    got, at = expert >= 0, expert.clamp(min=0).long()
    hit = torch.zeros_like(zd).scatter_add(1, at, got.double())
    for sigmoid, renormalize in ((False, True), (True, True), (False, False), (True, False)):
        dz = torch.full_like(z, math.nan)
        ops.sp_route_backward(z, expert, dw, dz, sigmoid=sigmoid, renormalize=renormalize, scale=1.5)
        up = torch.zeros_like(zd).scatter_add(1, at, torch.where(got, 1.5 * dw.double(), 0.0))
        s = torch.sigmoid(zd) if sigmoid else torch.softmax(torch.where(zd > -INF, zd, -1e6), 1) * (zd > -INF)
        total = (s * hit).sum(1, keepdim=True)
        if renormalize:
            up = torch.where(total > 0, hit * (up - (up * s).sum(1, keepdim=True) / total) / total, 0.0)
        # (renormalised weights do not change with the sum of all)
        want = up * s * (1 - s) if sigmoid else s * up if renormalize else s * (up - (up * s).sum(1, keepdim=True))
        want = torch.where(got.any(1, keepdim=True), want, 0.0)
        # as in the test of few rows: shares are off by (2 (spread + 8) + 36) u, softmax scores by less than (3 spread + 60) u, spread that of the
        # row's logits; the sum over the chosen is one of 32 products; the formula in 64 bits by 2^-49 of the size of what it is made of
        zf = torch.where(zd > -INF, zd, 0.0)
        rel = 3 * (zf.amax(1, keepdim=True) - zf.amin(1, keepdim=True)) + 120
        mag = torch.where(got, 1.5 * dw.double().abs(), 0.0).sum(1, keepdim=True)
        size = hit * s if sigmoid and not renormalize else hit if renormalize else s + hit * s
        bound = rel * U * mag * size * 2 + half_step(torch, t) * want.abs() * 1.01 + 2.0 ** -49 * mag + 1e-37
        assert_within(torch, dz, want, bound, ("dz", sigmoid, renormalize))
    ops.sp_ops_check()


# 32768 rows of 64 pieces of 16 bytes at once, 524288 of 4
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,bytes_,top", [(40001, 1024, 3), (33001, 1028, 1), (530001, 64, 2), (40001, 1024, 9)])
def test_dispatch_and_combine_of_many_rows(gpu, ops, n, bytes_, top, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    d = bytes_ // (4 if dtype == "f32" else 2)
    g = torch.Generator(device=DEV).manual_seed(n + d)
    place = torch.randperm(n * top, device=DEV, generator=g).int().view(n, top)
    place[torch.rand(n, top, device=DEV, generator=g) < 0.1] = -1
    here, at = place >= 0, place.clamp(min=0).long()
    x = torch.randn(n, d, device=DEV, generator=g).to(t)
    xs = torch.full((n * top, d), 5.0, dtype=t, device=DEV)
    ops.sp_dispatch(x, place, xs)
    want = torch.full_like(xs, 5.0)
    for j in range(top):
        want[at[:, j][here[:, j]]] = x[here[:, j]]
    assert torch.equal(xs, want)
    ys, r = torch.randn(n * top, d, device=DEV, generator=g).to(t), torch.randn(n, d, device=DEV, generator=g).to(t)
    weight = torch.randn(n, top, device=DEV, generator=g)
    y = torch.full_like(x, math.nan)
    ops.sp_combine(ys, place, y, weight=weight, residual=r)
    total, size = r.double(), r.double().abs()
    for j in range(top):
        part = torch.where(here[:, j, None], ys[at[:, j]].double(), 0.0) * weight[:, j, None].double()
        total, size = total + part, size + part.abs()
    bound = (top + 2) * U * size
    assert_within(torch, y, total, bound + half_step(torch, t) * (total.abs() + bound) + 1e-38, "y")
    dy, dys, dweight = x, torch.full_like(ys, 5.0), torch.full((n, top), math.nan, device=DEV)
    ops.sp_combine_backward(dy, ys, place, weight, dys=dys, dweight=dweight)
    want.fill_(5.0)
    for j in range(top):
        full = (dy.float() * weight[:, j, None]).to(t)
        want[at[:, j][here[:, j]]] = full[here[:, j]]
        products = torch.where(here[:, j, None], ys[at[:, j]].double(), 0.0) * dy.double()
        assert_within(torch, dweight[:, j], products.sum(1), (d + 8) * U * products.abs().sum(1) + 1e-38, ("dweight", j))
    assert torch.equal(dys, want)
    ops.sp_ops_check()


def numbers(torch, n, d, seed, offset):
    """The 16-bit numbers of sp_dropout, all rows at once: Philox in 64-bit words, whose low 64 bits are right whatever the sign."""
    low = 0xFFFFFFFF
    piece = torch.arange((d + 7) // 8, device=DEV).expand(n, -1)
    row = torch.arange(n, device=DEV)[:, None].expand_as(piece)
    c = [piece, row, torch.full_like(piece, offset & low), torch.full_like(piece, offset >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & low) ^ c[1] ^ k[0], b & low, (a >> 32 & low) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    words = torch.stack(c, 2)
    return torch.stack([words & 0xFFFF, words >> 16], 3).view(n, -1)[:, :d]


# pieces of eight columns whose workgroups of 256 lie inside a row, across some, or across 256 rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(60001, 77), (60001, 80), (301, 16390), (2100, 2056), (530001, 8), (530001, 5), (1000003, 9), (8, 524301)])
def test_dropout_of_many_pieces(gpu, ops, n, d, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    g = torch.Generator(device=DEV).manual_seed(n + d)
    p, seed, offset = 0.3, 2 ** 63 + 12345, 2 ** 40 + 3
    number = numbers(torch, n, d, seed, offset)
    for i, j in ((0, 0), (n - 1, d - 1), (n // 2, d // 3)):
        words = philox((j // 8, i, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        assert int(number[i, j]) == words[j % 8 // 2] >> 16 * (j % 2) & 0xFFFF
    drop = round(p * 65536)
    kept = number >= drop
    for layout, with_r in (("plain", False), ("odd", True), ("apart", True)):
        x = in_layout(torch, torch.randn(n, d, device=DEV, generator=g).to(t), layout)
        r = in_layout(torch, torch.randn(n, d, device=DEV, generator=g).to(t), layout) if with_r else None
        y = in_layout(torch, torch.full((n, d), math.nan, dtype=t, device=DEV), layout)
        ops.sp_dropout(x, y, p, seed, offset=offset, residual=r)
        part = torch.where(kept, x.double() / (1 - drop / 65536), 0.0)
        want = part + (0.0 if r is None else r.double())
        bound = 2 * U * part.abs() + U * want.abs()
        assert_within(torch, y, want, bound + half_step(torch, t) * (want.abs() + bound), "y")
        same = in_layout(torch, x, layout)
        ops.sp_dropout(same, same, p, seed, offset=offset, residual=r)
        assert torch.equal(same, y)
        if r is not None:
            ops.sp_dropout(x, r, p, seed, offset=offset, residual=r)
            assert torch.equal(r, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_of_more_than_32_bits_of_pieces(gpu, ops, dtype):
    """Three pieces to a row, 4.35e9 in all, in place; 50 or 100 GB."""
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    torch.cuda.empty_cache()
    n, d, p = 1450000000, 17, 0.3
    x = torch.ones(n * d, dtype=t, device=DEV).view(n, d)
    ops.sp_dropout(x, x, p, 99, offset=5)
    drop = round(p * 65536)
    kept = torch.tensor(65536.0 / (65536 - drop)).to(t)
    edge = 2 ** 32 // 3                                    # the row that holds piece 2^32
    for first in (0, 7 * 10 ** 8, edge - 3, n - 100):
        for i in range(first, first + 6):
            words = [philox((piece, i, 5, 0), (99, 0)) for piece in range(3)]
            want = [words[c // 8][c % 8 // 2] >> 16 * (c % 2) & 0xFFFF >= drop for c in range(d)]
            assert torch.equal(x[i], torch.where(torch.tensor(want, device=DEV), kept.to(DEV), 0.0).to(t)), i
    # and all of the others: kept or dropped, nothing untouched
    for part in x.view(-1).split(1 << 30):
        assert bool(((part == 0) | (part == kept.to(DEV))).all())
    del x, part
    torch.cuda.empty_cache()


# 32768 rows of a wavefront each at once, 8192 of a workgroup each, 4096 of those that are read twice
@pytest.mark.parametrize("n,d,dtype", [(40001, 512, "bf16"), (40001, 250, "f32"), (9001, 4096, "bf16"), (9001, 8200, "bf16"), (8300, 4100, "f32"), (4200, 32776, "bf16")])
def test_quantize_many_rows(gpu, ops, n, d, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    g = torch.Generator(device=DEV).manual_seed(n + d)
    # every row of its own size, so that a row's largest value is no other's
    x = (torch.randn(n, d, device=DEV, generator=g) * torch.exp2(torch.randint(-20, 20, (n, 1), device=DEV, generator=g).float())).to(t)
    x[:: 13] = 0.0
    x[4:: 17, d // 2] = math.nan
    q, scale = torch.full((n, d), 99, dtype=torch.int8, device=DEV), torch.full((n,), -1.0, device=DEV)
    ops.sp_quantize_rows(x, q, scale)
    high = x.float().abs().amax(1, keepdim=True)
    fine = torch.isfinite(high)
    # the definition's float32, on the host; a quotient of two tensors, since a number over a tensor is rounded twice
    high, fine = high.cpu(), fine.cpu()
    most = torch.full_like(high, 127.0)
    assert torch.equal(scale.cpu().nan_to_num(-2.0), torch.where(fine, high / most, -2.0)[:, 0])
    by = torch.where(fine & (high > 0), most / high, 0.0).to(DEV)
    want = torch.where(by > 0, torch.round(x.float() * by), 0.0).nan_to_num(0.0).to(torch.int8)
    assert torch.equal(q, want)
