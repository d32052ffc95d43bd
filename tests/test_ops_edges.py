"""The operators that train the heads where their contract is easily missed: ends of the ranges, values that are no numbers, empty
batches, tensors that change under a caller's list."""
import math

import numpy as np
import pytest

from tests.test_ops import DEV, U, assert_within, dtype_of, gpu, half_step, offsets_of, ops, plain_linear, plain_linear_backward

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
