"""The ends of the ranges of the operators for heads that are made of experts, on the GPU, against their definitions in 64 bits."""
import math

import numpy as np
import pytest

from tests.test_experts import DEV, INF, U, assert_within, dtype_of, gpu, half_step, in_layout, ops, quantized_layer  # noqa: F401 (fixtures)

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
