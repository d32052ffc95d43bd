"""What binding.Ops turns down of the operators for heads that are made of experts, on the CPU: nothing is launched, and there is no handle."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2505_06641_amd import binding, build


@pytest.fixture(scope="module")
def calls():
    if not os.path.exists(build.NATIVE):
        build.build_library(verbose=False)
    return binding.load_native().OpsBase()


def test_the_gradient_of_the_weights_needs_the_rows(calls):
    dy, place, dweight = torch.zeros(3, 4), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    for kw in (dict(dweight=dweight), dict(dweight=dweight, dys=torch.zeros(6, 4))):
        with pytest.raises(binding.SneakPeekError, match="ys is missing"):
            calls.sp_combine_backward(dy, None, place, **kw)
