"""The example that fits a head made of experts: it runs, and its gradients are those of its formulas in 64 bits."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need a real MI355X")
    import train_expert_heads
    return torch, train_expert_heads


@pytest.mark.parametrize("flags", [[], ["--bf16"]])
def test_it_runs(example, flags):
    torch, ex = example
    full, eight = ex.main(["--steps", "3"] + flags)
    assert full.shape == eight.shape == (4096, 10) and bool(torch.isfinite(full).all()) and bool(torch.isfinite(eight).all())


def test_its_gradients(example):
    torch, ex = example
    from tests.test_experts import kept_by_definition
    ops = ex.binding.Ops()
    n, d, hidden, classes, experts, top, p = 300, 40, 24, 7, 6, 2, 0.25
    g = torch.Generator().manual_seed(2)
    x, label = (2 * torch.randn(n, d, generator=g) + 0.5).cuda(), torch.randint(0, classes, (n,), generator=g).int().cuda()
    head = ex.ExpertHead(ops, n, d, hidden, classes, experts, top, torch.float32, seed=5, p=p)
    head.bias.copy_(0.05 * torch.randn(experts, generator=g))
    head.steps.fill_(3)
    got = {k: v.clone() for k, v in head.gradients(x, label).items()}
    ops.sp_ops_check()
    w = {k: v.double().cpu().requires_grad_() for k, v in head.weights.items()}
    x1 = torch.nn.functional.layer_norm(x.double().cpu(), (d,), w["gamma"], w["beta"], 1e-5)
    at, place = head.expert.cpu().long(), head.place.cpu().long()
    score = torch.sigmoid(x1 @ w["router"][0])
    # the experts are the best ones: no other has a larger score and bias, up to what 32 bits of the router's sums leave open
    value = score.detach() + head.bias.double().cpu()
    assert bool((value.gather(1, at).amin(1) >= value.scatter(1, at, -1.0).amax(1) - 1e-5).all())
    share = score.gather(1, at) / score.gather(1, at).sum(1, keepdim=True)
    kept = kept_by_definition(torch, n * top, hidden, p, 5, 3).cpu()
    h = torch.relu((x1[:, None, None, :] @ w["w1"][at]).squeeze(2) + w["b1"][at]) * kept[place] / (1 - p)
    ys = (h[:, :, None, :] @ w["w2"][at]).squeeze(2) + w["b2"][at]
    z = (x1 + (share[:, :, None] * ys).sum(1)) @ w["w"][0] + w["b"][0]
    torch.nn.functional.cross_entropy(z, label.cpu().long()).backward()
    # sums of at most 300 products in a chain of eight layers: 1e-5 of a gradient's norm is some ten times their roundings (24 half steps of 2^-24 a layer)
    # at random, and far below any part left out
    for k, v in w.items():
        off = float((got[k].double().cpu() - v.grad).norm() / v.grad.norm())
        assert math.isfinite(off) and off < 1e-5, (k, off)
    ops.close()
