"""Grouped linear layers at sizes that reach every kernel of theirs, against the definitions in 64 bits.

Few rows are computed in pieces of 16 rows, more of them in tiles of 128 rows by 64 or 128 columns with 256 or 512 threads, dW in tiles
of its own, with its group's rows in one piece or in chunks, alone or in the launch of dx.  `kernels` below says by sizes which of these a
call reaches; the first tests, which need no GPU, compare its constants with the source and see to it that nothing is left out.
"""
import math
import os
import re

import pytest

from paper_2505_06641_amd import build
from tests.test_ops import DEV, LINEAR_SIZES, U, assert_within, dtype_of, gpu, half_step, offsets_of, ops, plain_linear, plain_linear_backward

# rows of the groups, rows of no group, inputs, outputs: past the bounds of the few-row kernels for y and for dx
TILE_SIZES = [
    ((1500, 128, 0, 129, 1, 1300), 5, 230, 419),       # odd widths, groups of less than a tile, of one, of one and a row
    ((15000, 0, 5990, 1), 9, 136, 608),                # y: more than 768 tiles
    ((6000, 15000), 0, 608, 136),                      # dx: more than 768 tiles
    ((10001, 11000), 3, 70, 50),                       # y of up to 64 columns
    ((41000, 2, 777), 0, 33, 20),                      # dx of up to 64 columns, a depth shorter than a piece
    ((5000, 4000), 1, 257, 129),                       # a depth, and a last tile of columns, of one
    ((50000,), 0, 1, 3),                               # one input
    ((3000, 64, 4000), 2, 64, 512),                    # dW of up to 64 inputs
    ((300, 5, 0, 70) * 4, 0, 1024, 1000),              # dW: more than 768 tiles, every group's rows in one piece
    ((60000, 40000), 0, 130, 130),                     # dW: more than 768 tiles of chunks
    ((2000, 3000), 0, 2048, 2048),                     # dW: more sums than the workspace has room for in chunks
]

# ---------------------------------------------------------------- which kernels a call reaches

FEW_ROWS, FEW_COLS, FEW_DX_COLS, FEW_DX_DEPTH = 16, 32, 16, 128
WORKSPACE = 32 << 20


def ceil_div(a, b):
    return -(-a // b)


def row_tiles(n, groups, rows):
    return min(ceil_div(n, rows) + groups, (n + min(n, groups + 1) * (rows - 1)) // rows + 8)


def few(n, groups, width, cols, f32, depth):
    most = 2560 if f32 or (cols == FEW_DX_COLS and depth <= FEW_DX_DEPTH) else 1280
    return (ceil_div(n, FEW_ROWS) + min(n, groups)) * ceil_div(width, cols) <= most


def tiles(bm, bn, masked, count):
    threads = 512 if (bm, bn) == (128, 128) and (masked or count <= 768) else 256
    return f"{bm}x{bn}/{threads}"


def dw_chunk(n, groups, k, m, count, f32):
    stride = (k * m + m + 3) // 4 * 4
    chunk = int(math.sqrt(n * (8.0 * stride / 4e12) / (55e-9 if f32 else 19e-9)))
    lo = n * count // 2048
    chunk = min(max(chunk, lo), max(lo, n * count // 256))
    chunk = ceil_div(max(chunk, 64), 64) * 64
    most = WORKSPACE // (stride * 4) - groups
    if most <= 0:
        return 0
    chunk = max(chunk, ceil_div(n, most))
    return chunk if chunk < n else 0


def kernels(sizes, spare, k, m, f32, masked):
    """Of (y, dx and dW together, dx alone, dW alone); masked concerns the gradients."""
    n, groups = sum(sizes) + spare, len(sizes)
    y = "few" if few(n, groups, m, FEW_COLS, f32, k) else tiles(128, 64 if m <= 64 else 128, False,
                                                               row_tiles(n, groups, 128) * ceil_div(m, 64 if m <= 64 else 128))
    cols = 64 if k <= 64 else 128
    dx = "few" if few(n, groups, k, FEW_DX_COLS, f32, m) else tiles(128, cols, masked, row_tiles(n, groups, 128) * ceil_div(k, cols))
    bm, bn = 64 if k <= 64 else 128, 64 if m <= 64 else 128
    kt, mt = ceil_div(k, bm), ceil_div(m, bn)
    chunk = dw_chunk(n, groups, k, m, kt * mt, f32)
    count = (ceil_div(n, chunk) + groups if chunk else groups) * kt * mt
    how = "chunks" if chunk else "whole"
    dw = f"{tiles(bm, bn, masked, count)} {how}"
    both = f"{bm}x{bn} {how}" if dx == "few" and ceil_div(count, 8) * 8 <= 768 else None
    return y, both, dx, dw


def test_the_rule_is_the_sources():
    read = lambda name: open(os.path.join(build.CSRC, name)).read()
    ops_hip, few_h = read("sp_ops.hip"), read("sp_ops_linear_few.h")
    assert re.search(r"kFewRows = 16, kFewCols = 32, kFewThreads = 512;", few_h) and re.search(r"kFewDxCols = 16, kFewDxThreads = 256;", few_h)
    for line in ("(dtype == SP_F32 || (cols == kFewDxCols && depth <= kFewDxThreads / 64 * 32) ? 2560 : 1280)",
                 "((n + kFewRows - 1) / kFewRows + std::min(n, groups)) * ((width + cols - 1) / cols)",
                 "a.row_tiles * a.col_tiles <= 768", "few && dw && dw_blocks <= 768", "{ return k <= 64 ? 64 : 128; }", "{ return width <= 64 ? 64 : 128; }",
                 "sums = 8.0 * (double)chunk_stride(a) / 4e12, row = dtype == SP_F32 ? 55e-9 : 19e-9;",
                 "std::clamp<int64_t>(chunk, a.n * tiles / 2048, std::max<int64_t>(a.n * tiles / 2048, a.n * tiles / 256))",
                 "std::min((n + rows - 1) / rows + groups, (n + std::min(n, groups + 1) * (rows - 1)) / rows + kXcds)"):
        assert line in ops_hip, line
    binding = open(os.path.join(build.PKG, "binding.py")).read()
    assert "workspace_bytes: int = 32 << 20" in binding


@pytest.mark.parametrize("f32", [True, False])
def test_the_sizes_reach_every_kernel(f32):
    ys, boths, dxs, dws = set(), {True: set(), False: set()}, {True: set(), False: set()}, {True: set(), False: set()}
    for case in LINEAR_SIZES + TILE_SIZES:
        for masked in (True, False):
            y, both, dx, dw = kernels(*case, f32, masked)
            ys.add(y)
            boths[masked].add(both)
            dxs[masked].add(dx)
            dws[masked].add(dw)
    assert ys == {"few", "128x64/256", "128x128/512", "128x128/256"}
    assert dxs[True] == {"few", "128x64/256", "128x128/512"}
    assert dxs[False] == dxs[True] | {"128x128/256"}
    narrow = {f"{bm}x{bn}" for bm in (64, 128) for bn in (64, 128)}
    for masked in (True, False):
        assert {b.split()[0] for b in boths[masked] if b} == narrow and {b.split()[1] for b in boths[masked] if b} == {"chunks", "whole"}
        want = {f"{s}/256" for s in narrow if s != "128x128"} | {"128x128/512"} | (set() if masked else {"128x128/256"})
        assert {d.split()[0] for d in dws[masked]} == want and {d.split()[1] for d in dws[masked]} == {"chunks", "whole"}
    for case in TILE_SIZES[:6]:                               # these are here for the tiles of y and of dx
        y, _, dx, _ = kernels(*case, f32, False)
        assert y != "few" and dx != "few", case


# ---------------------------------------------------------------- values


class Rows:
    """[n, d] in one of three layouts, NaN around the rows; `intact` says whether that is still so."""

    def __init__(self, torch, g, n, d, t, layout, scale=1.0):
        pad, lead = {"plain": (0, 0), "apart": (16, 0), "odd": (3, 1)}[layout]
        self.store = torch.full((n * (d + pad) + lead + 1,), math.nan, dtype=t, device=DEV)
        grid = self.store[lead:lead + n * (d + pad)].view(n, d + pad)
        self.v, self.pad, self.ends = grid[:, :d], grid[:, d:], (self.store[:lead], self.store[lead + n * (d + pad):])
        if g is not None:
            self.v.copy_(torch.randn(n, d, device=DEV, generator=g) * scale)

    def intact(self):
        return bool(self.pad.isnan().all()) and all(bool(e.isnan().all()) for e in self.ends)


def weights(torch, g, groups, k, m, t, layout):
    w = (torch.randn(groups, k, m, device=DEV, generator=g) / math.sqrt(k)).to(t)
    if layout != "odd":
        return w
    store = torch.full((w.numel() + 2,), math.nan, dtype=t, device=DEV)      # at an element's alignment, NaN around them
    store[1:-1] = w.reshape(-1)
    return store[1:-1].view(w.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "bf16_to_f32"])
@pytest.mark.parametrize("sizes,spare,k,m", TILE_SIZES)
def test_grouped_linear_in_tiles(gpu, ops, sizes, spare, k, m, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype.split("_")[0])
    to = torch.float32 if dtype == "bf16_to_f32" else t
    n = sum(sizes) + spare
    g = torch.Generator(device=DEV).manual_seed(n * 31 + k * 7 + m)
    offsets = offsets_of(torch, sizes)
    for layout, extras in (("plain", ()), ("odd", ("bias", "relu", "residual", "act")), ("apart", ("bias", "residual")),
                           ("plain", ("bias", "relu", "residual", "act"))):
        x = Rows(torch, g, n, k, t, layout)
        x.v[n - spare:] = math.nan                           # rows of no group touch nothing
        w = weights(torch, g, len(sizes), k, m, t, layout)
        bias = torch.randn(len(sizes), m, device=DEV, generator=g) if "bias" in extras else None
        residual = Rows(torch, g, n, m, to, layout) if "residual" in extras else None
        y = Rows(torch, None, n, m, to, layout)
        act = Rows(torch, None, n, m, to, layout) if "act" in extras else None
        ops.sp_grouped_linear(x.v, offsets, w, y.v, bias=bias, relu="relu" in extras, residual=residual and residual.v, act_out=act and act.v)
        want, want_act, size = plain_linear(torch, x.v, sizes, w, bias, "relu" in extras, residual and residual.v)
        # a sum of k products, bias and residual; the products that a float32 factor's split leaves out are 1.001 u of theirs
        bound = (k + 10) * U * size + 1e-36
        assert_within(torch, y.v, want, bound + half_step(torch, to) * (want.abs() + bound), "y")
        assert y.intact()
        if act:
            assert_within(torch, act.v, want_act, bound + half_step(torch, to) * (want_act.abs() + bound), "act_out")
            assert act.intact()
        if residual:                                          # the sum may go where the residual was
            ops.sp_grouped_linear(x.v, offsets, w, residual.v, bias=bias, relu="relu" in extras, residual=residual.v)
            assert torch.equal(residual.v, y.v) and residual.intact()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,spare,k,m", TILE_SIZES)
def test_grouped_linear_backward_in_tiles(gpu, ops, sizes, spare, k, m, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    n, groups, longest = sum(sizes) + spare, len(sizes), max(sizes)
    g = torch.Generator(device=DEV).manual_seed(n * 37 + k * 11 + m)
    offsets = offsets_of(torch, sizes)
    for layout, masked in (("plain", True), ("odd", True), ("apart", False), ("odd", False)):
        x, dy = Rows(torch, g, n, k, t, layout), Rows(torch, g, n, m, t, layout)
        act = Rows(torch, g, n, m, t, layout) if masked else None
        if masked:
            act.v.clamp_(min=0)
        x.v[n - spare:] = math.nan
        dy.v[n - spare:] = math.nan
        w = weights(torch, g, groups, k, m, t, layout)
        dx = Rows(torch, None, n, k, t, layout)
        dw, db = torch.full((groups, k, m), math.nan, device=DEV), torch.full((groups, m), math.nan, device=DEV)
        mask = act and act.v
        ops.sp_grouped_linear_backward(dy.v, x.v, offsets, w, act=mask, dx=dx.v, dw=dw, db=db)
        wx, ww, wb, sx, sw, sb = plain_linear_backward(torch, dy.v, mask, x.v, sizes, w)
        bound = (m + 10) * U * sx + 1e-36
        assert_within(torch, dx.v, wx, bound + half_step(torch, t) * (wx.abs() + bound), "dx")
        assert dx.intact()
        assert_within(torch, dw, ww, (longest + 10) * U * sw + 1e-36, "dw")
        assert_within(torch, db, wb, (longest + 10) * U * sb + 1e-36, "db")
        # each product alone has the same bits
        one = Rows(torch, None, n, k, t, layout)
        ops.sp_grouped_linear_backward(dy.v, x.v, offsets, w, act=mask, dx=one.v)
        assert torch.equal(one.v, dx.v)
        one = torch.full_like(dw, math.nan)
        ops.sp_grouped_linear_backward(dy.v, x.v, offsets, w, act=mask, dw=one)
        assert torch.equal(one, dw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,spare,k,m", [TILE_SIZES[0], TILE_SIZES[1], TILE_SIZES[3]])
def test_no_number_leaves_its_row_column_and_group_in_tiles(gpu, ops, sizes, spare, k, m, dtype):
    torch, _ = gpu
    t = dtype_of(torch, dtype)
    n, groups = sum(sizes) + spare, len(sizes)
    g = torch.Generator(device=DEV).manual_seed(n + k + m)
    offsets = offsets_of(torch, sizes)
    x, dy = (torch.randn(n, d, device=DEV, generator=g).to(t) for d in (k, m))
    w = weights(torch, g, groups, k, m, t, "plain")
    last = max(i for i, s in enumerate(sizes) if s)           # the group of the last rows that have one
    end = n - spare

    def results():
        y, dx = torch.empty(n, m, dtype=t, device=DEV), torch.empty(n, k, dtype=t, device=DEV)
        dw, db = torch.empty(groups, k, m, device=DEV), torch.empty(groups, m, device=DEV)
        ops.sp_grouped_linear(x, offsets, w, y)
        ops.sp_grouped_linear_backward(dy, x, offsets, w, dx=dx, dw=dw, db=db)
        return y, dx, dw, db

    clean = results()
    bad_rows, bad_dys = (sizes[0] - 1, end - 1), (2, end - 1)
    x[bad_rows[0], k - 1], x[bad_rows[1], 0] = math.nan, math.inf
    w[0, k // 2, m - 1] = math.nan
    dy[bad_dys[0], 0], dy[bad_dys[1], m - 1] = -math.inf, math.nan
    y, dx, dw, db = results()
    rows = torch.arange(n, device=DEV)
    hit = (rows == bad_rows[0]) | (rows == bad_rows[1])
    assert not bool(y[hit].isfinite().any())
    rest = ~hit[:, None] & ~((rows < sizes[0])[:, None] & (torch.arange(m, device=DEV) == m - 1)[None])
    assert torch.equal(y[rest], clean[0][rest])
    assert not bool(y[:sizes[0], m - 1].isfinite().any())
    hit = (rows == bad_dys[0]) | (rows == bad_dys[1])
    assert not bool(dx[hit].isfinite().any())
    rest = ~hit[:, None] & ~((rows < sizes[0])[:, None] & (torch.arange(k, device=DEV) == k // 2)[None])
    assert torch.equal(dx[rest], clean[1][rest])
    spoilt = torch.zeros_like(dw, dtype=torch.bool)
    spoilt[0, k - 1], spoilt[last, 0], spoilt[0, :, 0], spoilt[last, :, m - 1] = True, True, True, True
    assert torch.equal(dw[~spoilt], clean[2][~spoilt]) and not bool(dw[spoilt].isfinite().any())
    spoilt = torch.zeros_like(db, dtype=torch.bool)
    spoilt[0, 0], spoilt[last, m - 1] = True, True
    assert torch.equal(db[~spoilt], clean[3][~spoilt]) and not bool(db[spoilt].isfinite().any())
