"""Fits a head that is made of experts on the GPU, then serves with its weights rounded to 8 bits.

    python examples/train_expert_heads.py [--bf16] [--steps 200]

Labelled feature rows go through

    x1 = layer norm of x
    r  = x1 R                                             the router: a logit for every expert
    x2 = x1 + sum over a row's experts of w_e (drop(relu(x1 W1_e + b1_e)) W2_e + b2_e)
    z  = x2 W + b                                         logits over the classes
    loss: softmax cross entropy

and back.  A row's experts are the `top` of the largest sigmoid(r) + bias, the weights w_e their sigmoids over the sum of them.  The bias has no gradient: after
every step it moves towards experts that had fewer rows than others.  Afterwards the experts' layers are rounded to 8 bits and their outputs compared.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import numpy as np
import torch

from paper_2505_06641_amd import binding
from train_heads import labelled_rows

DEV = "cuda:0"


class ExpertHead:
    """Weights, gradients and activations of the model above for n rows; float32 weights, computed with in `dtype`."""

    def __init__(self, ops, n, d, hidden, classes, experts, top, dtype, seed, p=0.1):
        self.ops, self.dtype, self.p, self.seed, self.n, self.top = ops, dtype, p, seed, n, top
        g = torch.Generator().manual_seed(seed)
        init = lambda *s: (torch.randn(*s, generator=g) * s[1] ** -0.5).to(DEV)
        zero = lambda *s: torch.zeros(*s, device=DEV)
        self.weights = dict(gamma=zero(d) + 1, beta=zero(d), router=init(1, d, experts), w1=init(experts, d, hidden), b1=zero(experts, hidden),
                            w2=init(experts, hidden, d), b2=zero(experts, d), w=init(1, d, classes), b=zero(1, classes))
        self.grads = {k: torch.empty_like(v) for k, v in self.weights.items()}
        self.clip_list, self.norm = binding.TensorList(self.grads.values()), zero(1)
        self.low = {k: v.to(dtype) for k, v in self.weights.items() if v.dim() == 3}
        self.bias = zero(experts)                            # balances the experts
        self.steps = torch.zeros(1, dtype=torch.int64, device=DEV)
        whole = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
        room = lambda rows, w, t=dtype: torch.zeros(rows, w, dtype=t, device=DEV)
        pairs = n * top
        self.all = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        self.expert, self.place, self.offsets = whole(n, top), whole(n, top), whole(experts + 1)
        self.weight, self.dweight = (room(n, top, torch.float32) for _ in range(2))
        self.x1, self.x2, self.dx2, self.dx1, self.dr_x = (room(n, d) for _ in range(5))
        self.r, self.dr, self.z, self.dz = room(n, experts), room(n, experts), room(n, classes, torch.float32), room(n, classes)
        self.xs, self.ys, self.dys, self.dxs = (room(pairs, d) for _ in range(4))
        self.h, self.hd, self.dhd, self.dh = (room(pairs, hidden) for _ in range(4))
        self.mean, self.rstd, self.loss = (torch.empty(n, device=DEV) for _ in range(3))

    def route(self, x):
        o, w = self.ops, self.weights
        o.sp_layer_norm(x, self.x1, gamma=w["gamma"], beta=w["beta"], mean=self.mean, rstd=self.rstd)
        o.sp_grouped_linear(self.x1, self.all, self.low["router"], self.r)
        o.sp_route(self.r, self.expert, self.weight, sigmoid=True, bias=self.bias)
        o.sp_route_order(self.expert, self.offsets, self.place)
        o.sp_dispatch(self.x1, self.place, self.xs)

    def logits(self, x, training=False):
        o, w = self.ops, self.weights
        self.route(x)
        o.sp_grouped_linear(self.xs, self.offsets, self.low["w1"], self.h, bias=w["b1"], relu=True)
        o.sp_dropout(self.h, self.hd, self.p if training else 0.0, self.seed, step=self.steps)
        o.sp_grouped_linear(self.hd, self.offsets, self.low["w2"], self.ys, bias=w["b2"])
        o.sp_combine(self.ys, self.place, self.x2, weight=self.weight, residual=self.x1)
        o.sp_grouped_linear(self.x2, self.all, self.low["w"], self.z, bias=w["b"])
        return self.z

    def gradients(self, x, label):
        o, g, n = self.ops, self.grads, self.n
        self.logits(x, training=True)
        o.sp_cross_entropy(self.z, label, self.loss, scale=1.0 / n, dlogits=self.dz)
        o.sp_grouped_linear_backward(self.dz, self.x2, self.all, self.low["w"], dx=self.dx2, dw=g["w"], db=g["b"])
        o.sp_combine_backward(self.dx2, self.ys, self.place, self.weight, dys=self.dys, dweight=self.dweight)
        o.sp_grouped_linear_backward(self.dys, self.hd, self.offsets, self.low["w2"], dx=self.dhd, dw=g["w2"], db=g["b2"])
        o.sp_dropout(self.dhd, self.dh, self.p, self.seed, step=self.steps)
        o.sp_grouped_linear_backward(self.dh, self.xs, self.offsets, self.low["w1"], act=self.h, dx=self.dxs, dw=g["w1"], db=g["b1"])
        o.sp_combine(self.dxs, self.place, self.dx1, residual=self.dx2)        # the dispatch's gradient, and the residual's
        o.sp_route_backward(self.r, self.expert, self.dweight, self.dr, sigmoid=True)
        o.sp_grouped_linear_backward(self.dr, self.x1, self.all, self.low["router"], dx=self.dr_x, dw=g["router"])
        self.dx1 += self.dr_x
        o.sp_layer_norm_backward(self.dx1, x, self.mean, self.rstd, gamma=self.weights["gamma"], dgamma=g["gamma"], dbeta=g["beta"])
        return g

    def step(self, x, label, rate, max_norm):
        self.gradients(x, label)
        self.ops.sp_clip_grad_norm(self.clip_list, max_norm, self.norm)
        for k, v in self.weights.items():
            v.add_(self.grads[k], alpha=-rate)
            if k in self.low:
                self.low[k].copy_(v)
        rows = self.offsets.diff().float()
        self.bias.add_(torch.sign(rows.mean() - rows), alpha=0.001)
        self.steps.add_(1)                                   # the next step's mask is another one

    def round_to_8_bits(self):
        """The experts' layers for serving: an output's inputs next to each other, whole numbers and scales."""
        self.eight = {}
        for k in ("w1", "w2"):
            groups, inputs, outputs = self.weights[k].shape
            rows = self.weights[k].transpose(1, 2).reshape(groups * outputs, inputs).contiguous()
            q, scale = torch.empty(rows.shape, dtype=torch.int8, device=DEV), torch.empty(groups * outputs, device=DEV)
            self.ops.sp_quantize_rows(rows, q, scale)
            self.eight[k] = q.view(groups, outputs, inputs), scale.view(groups, outputs)

    def serve(self, x):
        """The logits with the experts' layers in 8 bits."""
        o, w = self.ops, self.weights
        self.route(x)
        for rows, k, b, out, relu in ((self.xs, "w1", "b1", self.h, True), (self.h, "w2", "b2", self.ys, False)):
            q, scale = torch.empty(rows.shape, dtype=torch.int8, device=DEV), torch.empty(rows.shape[0], device=DEV)
            o.sp_quantize_rows(rows, q, scale)
            o.sp_grouped_linear_quantized(q, scale, self.offsets, *self.eight[k], out, bias=w[b], relu=relu)
        o.sp_combine(self.ys, self.place, self.x2, weight=self.weight, residual=self.x1)
        o.sp_grouped_linear(self.x2, self.all, self.low["w"], self.z, bias=w["b"])
        return self.z


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--bf16", action="store_true")
    p.add_argument("--steps", type=int, default=200)
    args = p.parse_args(argv)
    n, d, hidden, classes, experts, top = 4096, 128, 64, 10, 16, 2
    dtype = torch.bfloat16 if args.bf16 else torch.float32
    x, _, label, _ = labelled_rows(np.random.default_rng(0), (n,), (classes,), d)
    x, label = torch.from_numpy(x).to(DEV).to(dtype), torch.from_numpy(label).to(DEV)
    ops = binding.Ops()
    head = ExpertHead(ops, n, d, hidden, classes, experts, top, dtype, seed=1)
    for step in range(args.steps):
        head.step(x, label, rate=0.5, max_norm=1.0)
        if step % 20 == 0 or step == args.steps - 1:
            rows = head.offsets.diff()
            print(f"step {step:4d}: mean loss {float(head.loss.mean()):.4f}, norm of all gradients {float(head.norm):.3f}, rows of an expert {int(rows.min())} to "
                  f"{int(rows.max())}", flush=True)
    ops.sp_ops_check()
    full = head.logits(x).clone()
    head.round_to_8_bits()
    eight = head.serve(x)
    ops.sp_ops_check()
    share = lambda z: float((z.argmax(1) == label).float().mean())
    print(f"accuracy {share(full):.3f}, with the experts in 8 bits {share(eight):.3f}; logits differ by {float((full - eight).norm() / full.norm()):.4f} of their norm")
    ops.close()
    return full, eight


if __name__ == "__main__":
    main()
