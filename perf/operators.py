"""What is measured of the operators that train the heads: grouped linear layers, layer norm, the loss and clipping.

A head is a small classifier of one application.  All applications' heads are trained together: the rows of a batch
are sorted by application, so that application a owns the rows offsets[a] .. offsets[a + 1], and every operator takes
all of them in one call.  `do` says which operator a case calls:

  linear         y = act(x W_a + b_a) + residual, rows grouped by application
  linear_back    its gradients with respect to rows, weights and biases
  norm           layer norm of every row
  norm_back      its gradients with respect to rows, gain and shift
  loss           softmax cross entropy over each application's own classes, with the gradient of the logits (`wide_out`: of
                 float32 logits of a bfloat16 head, whose backward pass takes bfloat16 gradients)
  clip           the norm over all gradients of a model, and the gradients scaled to at most that norm
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5


def _case(name, **kw):
    c = dict(do="linear", bf16=False, n=1, apps=1, skew=0.0, k=1, m=1, bias=True, relu=False, residual=False, wide_out=False,
             dx=True, ignored=0.0, weighted=False, tensors=1, elements=1, odd=False, max_norm=1.0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request of one of eight applications through a hidden layer: latency is all that counts
        _case("linear_one_request", bf16=True, n=1, apps=8, k=512, m=256, relu=True),
        # an adapter of wide embeddings: twelve applications of very different shares, y = x + relu(x W + b)
        _case("linear_adapter_bf16", bf16=True, n=100003, apps=12, skew=1.0, k=768, m=768, relu=True, residual=True),
        # logits of float32 logistic heads of 32 applications with up to 1000 classes
        _case("linear_logits_f32", n=262144, apps=32, k=256, m=1000),
        # a step on the three small float32 applications: the hidden layer's gradients
        _case("linear_back_small_f32", do="linear_back", n=4096, apps=3, skew=0.8, k=128, m=64, relu=True),
        # a step on eight applications with bfloat16 MLP heads: the hidden layer's gradients
        _case("linear_back_64k_bf16", do="linear_back", bf16=True, n=65536, apps=8, k=512, m=256, relu=True),
        # features of one scheduling window of an edge server
        _case("norm_window_bf16", do="norm", bf16=True, n=24, k=512),
        # features of the largest queue
        _case("norm_1m_f32", do="norm", n=1048576, k=256),
        # a step on wide embeddings
        _case("norm_back_64k_bf16", do="norm_back", bf16=True, n=65536, k=768),
        # a step on the three small applications: 10, 6 and 5 classes, some requests without a label
        _case("loss_small_f32", do="loss", n=4096, apps=3, skew=0.8, m=10, ignored=0.1),
        # a step on 32 applications of up to 1000 classes, weighted requests
        _case("loss_1000_f32", do="loss", n=131072, apps=32, skew=0.5, m=1000, weighted=True),
        # weights, biases, gain and shift of three small heads
        _case("clip_small", do="clip", tensors=14, elements=28000, odd=True),
        # many heads of many sizes
        _case("clip_many", do="clip", tensors=600, elements=120000000, odd=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw(rng):
    do = rng.choice(["linear", "linear", "linear_back", "linear_back", "norm", "norm_back", "loss", "clip"])
    bf16 = rng.random() < 0.5
    apps = _log_int(rng, 1, 32)
    skew = rng.choice([0.0, 0.5, 1.0])
    if do in ("linear", "linear_back"):
        # half of the widths are multiples of 32, as configurations have them, the others are any number
        k, m = ((_log_int(rng, 1, 32) * 32) if rng.random() < 0.5 else _log_int(rng, 3, 1024) for _ in range(2))
        relu = rng.random() < 0.5
        c = dict(do=do, bf16=bf16, n=_log_int(rng, 1, 262144), apps=apps, skew=skew, k=k, m=m, relu=relu)
        if do == "linear":
            c.update(bias=rng.random() < 0.8, residual=rng.random() < 0.4, wide_out=bf16 and rng.random() < 0.3)
        else:
            c.update(dx=rng.random() < 0.7)
        return c
    if do in ("norm", "norm_back"):
        k = _log_int(rng, 1, 64) * 32 if rng.random() < 0.5 else _log_int(rng, 3, 4096)
        return dict(do=do, bf16=bf16, n=_log_int(rng, 1, 1048576), k=k)
    if do == "loss":
        return dict(do=do, bf16=bf16, wide_out=bf16 and rng.random() < 0.5, n=_log_int(rng, 1, 262144), apps=apps, skew=skew,
                    m=_log_int(rng, 2, 4000), ignored=rng.choice([0.0, 0.1]), weighted=rng.random() < 0.5)
    tensors = _log_int(rng, 1, 600)
    return dict(do=do, tensors=tensors, elements=tensors * _log_int(rng, 10, 200000), odd=rng.random() < 0.7,
                max_norm=rng.choice([1.0, 1e6]))


def draw(rng):
    most = [work(c) for c in listed()]
    bytes_, flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        c = _case(None, **_draw(rng))
        w = work(c)
        if w["bytes"] <= bytes_ and w["flops"] <= flops:
            return c


def _sizes(n, apps, skew):
    """Rows of each application: shares proportional to (a + 1)^-skew, remainders to the first ones (few rows leave
    the last applications without any)."""
    share = [(a + 1.0) ** -skew for a in range(apps)]
    out = [int(n * s / sum(share)) for s in share]
    for i in range(n - sum(out)):
        out[i % apps] += 1
    return out


def _classes(case):
    """Classes of each application: the first one has the most, the others fewer."""
    return [max(2, int(case["m"] * (1.0 - 0.6 * a / case["apps"]))) if a else case["m"] for a in range(case["apps"])]


def _tensor_sizes(case):
    t, total = case["tensors"], case["elements"]
    if not case["odd"]:
        return [total // t] * t
    share = [1.0 / (1 + i % 7) ** 2 for i in range(t)]
    return [max(1, int(total * s / sum(share)) | 1) for s in share]


def _flat(tensors):
    """One buffer with room for all of them, as an optimizer keeps its gradients, and each one's view of it."""
    flat = torch.empty(sum(v.numel() for v in tensors), device=DEV)
    return flat, list(flat.split([v.numel() for v in tensors]))


def work(case):
    do, n, k, m = case["do"], case["n"], case["k"], case["m"]
    e = 2 if case["bf16"] else 4
    if do in ("linear", "linear_back"):
        sizes = _sizes(n, case["apps"], case["skew"])
        held = sum(1 for s in sizes if s)
        if do == "linear":
            out = 4 if case["wide_out"] else e
            b = n * k * e + held * k * m * e + n * m * out * (2 if case["residual"] else 1) + (held * m * 4 if case["bias"] else 0)
            return {"bytes": b + 4 * (case["apps"] + 1), "flops": 2 * n * k * m}
        b = n * k * e + n * m * e * (2 if case["relu"] else 1) + case["apps"] * (k + 1) * m * 4 + 4 * (case["apps"] + 1)
        if case["dx"]:
            b += n * k * e + held * k * m * e
        return {"bytes": b, "flops": (4 if case["dx"] else 2) * n * k * m}
    if do == "norm":
        return {"bytes": 2 * n * k * e + 8 * k + 8 * n, "flops": 8 * n * k}
    if do == "norm_back":
        return {"bytes": 3 * n * k * e + 12 * k + 8 * n, "flops": 13 * n * k}
    if do == "loss":
        sizes, classes = _sizes(n, case["apps"], case["skew"]), _classes(case)
        read = sum(s * c for s, c in zip(sizes, classes))
        return {"bytes": read * (4 if case["wide_out"] else e) + n * m * e + n * (16 if case["weighted"] else 12), "flops": 6 * read}
    total = sum(_tensor_sizes(case))
    return {"bytes": 8 * total, "flops": 3 * total}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    do, n, k, m, apps = case["do"], case["n"], case["k"], case["m"], case["apps"]
    t = torch.bfloat16 if case["bf16"] else torch.float32

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, device=DEV, generator=g) * scale).to(dtype)

    s = dict(case=case)
    if do in ("linear", "linear_back", "loss"):
        sizes = _sizes(n, apps, case["skew"])
        turn = seed % apps                    # which application owns the most rows changes with the seed
        sizes = sizes[turn:] + sizes[:turn]
        ends = [0]
        for v in sizes:
            ends.append(ends[-1] + v)
        s["ends"] = ends
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEV)
    if do == "linear":
        s["x"] = normal(n, k)
        s["w"] = normal(apps, k, m, scale=math.sqrt(2.0 / k))
        s["b"] = normal(apps, m, scale=0.1, dtype=torch.float32) if case["bias"] else None
        out = torch.float32 if case["wide_out"] else t
        s["r"] = normal(n, m, dtype=out) if case["residual"] else None
        s["out"] = out
        if own:
            s["y"] = torch.empty(n, m, dtype=out, device=DEV)
    elif do == "linear_back":
        s["x"] = normal(n, k)
        s["w"] = normal(apps, k, m, scale=math.sqrt(2.0 / k))
        s["dy"] = normal(n, m, scale=1.0 / max(1, n) ** 0.5)
        s["act"] = normal(n, m).clamp_(min=0) if case["relu"] else None
        if own:
            s["dx"] = torch.empty(n, k, dtype=t, device=DEV) if case["dx"] else None
            s["dw"] = torch.empty(apps, k, m, device=DEV)
            s["db"] = torch.empty(apps, m, device=DEV)
    elif do in ("norm", "norm_back"):
        shift = normal(n, 1, dtype=torch.float32)
        s["x"] = (torch.randn(n, k, device=DEV, generator=g).mul_(3.0).add_(shift)).to(t)
        s["gamma"] = 1.0 + normal(k, scale=0.1, dtype=torch.float32)
        s["beta"] = normal(k, scale=0.1, dtype=torch.float32)
        if do == "norm_back":
            # what the forward pass handed out: the statistics of these rows
            s["dy"] = normal(n, k)
            s["mean"] = torch.empty(n, device=DEV)
            s["rstd"] = torch.empty(n, device=DEV)
            for lo in range(0, n, 65536):
                x = s["x"][lo:lo + 65536].double()
                mean = x.mean(1, keepdim=True)
                s["mean"][lo:lo + 65536] = mean[:, 0]
                s["rstd"][lo:lo + 65536] = ((x - mean).square().mean(1) + EPS).rsqrt()
            if own:
                s["dx"], s["dgamma"], s["dbeta"] = torch.empty_like(s["x"]), torch.empty(k, device=DEV), torch.empty(k, device=DEV)
        elif own:
            s["y"], s["mean"], s["rstd"] = torch.empty_like(s["x"]), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    elif do == "loss":
        classes = _classes(case)
        s["logits"] = normal(n, m, scale=2.0, dtype=torch.float32 if case["wide_out"] else t)
        s["out"] = t
        s["app"] = torch.repeat_interleave(torch.arange(apps, dtype=torch.int32, device=DEV), torch.tensor(sizes, device=DEV))
        s["n_classes"] = torch.tensor(classes, dtype=torch.int32, device=DEV)
        u = torch.rand(n, device=DEV, generator=g)
        s["label"] = (u * s["n_classes"][s["app"].long()]).int()
        if case["ignored"]:
            s["label"][torch.rand(n, device=DEV, generator=g) < case["ignored"]] = -1
        s["weight"] = torch.rand(n, device=DEV, generator=g) if case["weighted"] else None
        s["scale"] = 1.0 / n
        if own:
            s["loss"], s["dlogits"] = torch.empty(n, device=DEV), torch.empty(n, m, dtype=t, device=DEV)
    else:
        s["grads"] = [normal(v, scale=0.02, dtype=torch.float32) for v in _tensor_sizes(case)]
        if own:
            s["flat"], s["clipped"] = _flat(s["grads"])
            s["norm"] = torch.empty(1, device=DEV)
    if own:
        from paper_2505_06641_amd import binding
        s["ops"] = binding.Ops()
        if do == "clip":                      # a training program's gradients stay where they are: it keeps the list of them
            s["list"] = binding.TensorList(s["grads"], out=s["clipped"])
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    ops, case, do = s["ops"], s["case"], s["case"]["do"]
    if do == "linear":
        ops.sp_grouped_linear(s["x"], s["offsets"], s["w"], s["y"], bias=s["b"], relu=case["relu"], residual=s["r"])
        return s["y"]
    if do == "linear_back":
        ops.sp_grouped_linear_backward(s["dy"], s["x"], s["offsets"], s["w"], act=s["act"], dx=s["dx"], dw=s["dw"], db=s["db"])
        return s["dx"], s["dw"], s["db"]
    if do == "norm":
        ops.sp_layer_norm(s["x"], s["y"], gamma=s["gamma"], beta=s["beta"], eps=EPS, mean=s["mean"], rstd=s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if do == "norm_back":
        ops.sp_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], gamma=s["gamma"], dx=s["dx"], dgamma=s["dgamma"],
                                   dbeta=s["dbeta"])
        return s["dx"], s["dgamma"], s["dbeta"]
    if do == "loss":
        ops.sp_cross_entropy(s["logits"], s["label"], s["loss"], app=s["app"], n_classes=s["n_classes"], weight=s["weight"],
                             scale=s["scale"], dlogits=s["dlogits"])
        return s["loss"], s["dlogits"]
    ops.sp_clip_grad_norm(s["list"], case["max_norm"], s["norm"])
    return s["norm"], s["flat"]


def _plain(s):
    case, do = s["case"], s["case"]["do"]
    if do == "linear":
        y = torch.empty(case["n"], case["m"], dtype=s["out"], device=DEV)
        for a in range(case["apps"]):
            lo, hi = s["ends"][a], s["ends"][a + 1]
            if lo == hi:
                continue
            z = s["x"][lo:hi].float() @ s["w"][a].float()
            if s["b"] is not None:
                z = z + s["b"][a]
            if case["relu"]:
                z = torch.where(z < 0, 0.0, z)
            if s["r"] is not None:
                z = z + s["r"][lo:hi].float()
            y[lo:hi] = z
        return y
    if do == "linear_back":
        x, dy = s["x"].float(), s["dy"].float()
        dz = dy if s["act"] is None else torch.where(s["act"] > 0, dy, 0.0)
        dx = torch.empty(case["n"], case["k"], dtype=s["x"].dtype, device=DEV) if case["dx"] else None
        dw = torch.zeros(case["apps"], case["k"], case["m"], device=DEV)
        db = torch.zeros(case["apps"], case["m"], device=DEV)
        for a in range(case["apps"]):
            lo, hi = s["ends"][a], s["ends"][a + 1]
            if lo == hi:
                continue
            if case["dx"]:
                dx[lo:hi] = dz[lo:hi] @ s["w"][a].float().t()
            dw[a] = x[lo:hi].t() @ dz[lo:hi]
            db[a] = dz[lo:hi].sum(0)
        return dx, dw, db
    if do == "norm":
        x = s["x"].float()
        mean = x.sum(1, keepdim=True) / case["k"]
        d = x - mean
        rstd = 1.0 / torch.sqrt((d * d).sum(1, keepdim=True) / case["k"] + EPS)
        y = d * rstd * s["gamma"] + s["beta"]
        return y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]
    if do == "norm_back":
        x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        gy = dy * s["gamma"]
        dx = rstd * (gy - gy.sum(1, keepdim=True) / case["k"] - xh * ((gy * xh).sum(1, keepdim=True) / case["k"]))
        return dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)
    if do == "loss":
        z = s["logits"].float()
        inside = torch.arange(case["m"], device=DEV)[None, :] < s["n_classes"][s["app"].long()][:, None]
        z = torch.where(inside, z, float("-inf"))
        top = z.max(1, keepdim=True).values
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        counted = s["label"] >= 0
        at = s["label"].clamp(min=0).long()[:, None]
        w = counted.float() if s["weight"] is None else s["weight"] * counted
        loss = (torch.log(total) + top - z.gather(1, at))[:, 0] * w
        hit = torch.arange(case["m"], device=DEV)[None, :] == at
        grad = (e / total - hit.float()) * (w * s["scale"])[:, None]
        return loss, grad.to(s["out"])
    total = torch.zeros(1, dtype=torch.float64, device=DEV)
    for v in s["grads"]:
        total += (v.double() * v.double()).sum()
    norm = torch.sqrt(total)
    c = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0).float()
    flat, clipped = _flat(s["grads"])
    for v, o in zip(s["grads"], clipped):
        torch.mul(v, c, out=o)
    return norm.float(), flat


def exact(case, seed):
    """The operators' values in 64 bits, from their definitions."""
    s = prepare(case, seed)
    do, f64 = case["do"], torch.float64
    if do == "linear":
        out = torch.empty(case["n"], case["m"], dtype=f64, device=DEV)
        for a, (lo, hi) in enumerate(zip(s["ends"], s["ends"][1:])):
            z = torch.mm(s["x"][lo:hi].to(f64), s["w"][a].to(f64))
            if case["bias"]:
                z += s["b"][a].to(f64)
            if case["relu"]:
                z.clamp_(min=0)
            if case["residual"]:
                z += s["r"][lo:hi].to(f64)
            out[lo:hi] = z
        return out
    if do == "linear_back":
        dx = torch.empty(case["n"], case["k"], dtype=f64, device=DEV) if case["dx"] else None
        dw = torch.empty(case["apps"], case["k"], case["m"], dtype=f64, device=DEV)
        db = torch.empty(case["apps"], case["m"], dtype=f64, device=DEV)
        for a, (lo, hi) in enumerate(zip(s["ends"], s["ends"][1:])):
            dz = s["dy"][lo:hi].to(f64)
            if case["relu"]:
                dz *= s["act"][lo:hi].to(f64).gt(0)
            if case["dx"]:
                torch.mm(dz, s["w"][a].to(f64).t(), out=dx[lo:hi])
            torch.mm(s["x"][lo:hi].to(f64).t(), dz, out=dw[a])
            torch.sum(dz, 0, out=db[a])
        return dx, dw, db
    if do == "norm":
        x = s["x"].to(f64)
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = (var + EPS).rsqrt()
        y = torch.addcmul(s["beta"].to(f64), (x - mean) * rstd, s["gamma"].to(f64))
        return y, mean[:, 0], rstd[:, 0]
    if do == "norm_back":
        # the statistics are inputs; with them fixed, dx is the gradient projected off the row's constant and its xh
        step = 1 << 16
        dx = torch.empty(case["n"], case["k"], dtype=f64, device=DEV)
        dgamma = torch.zeros(case["k"], dtype=f64, device=DEV)
        dbeta = torch.zeros(case["k"], dtype=f64, device=DEV)
        for lo in range(0, case["n"], step):
            rows = slice(lo, lo + step)
            dy, r = s["dy"][rows].to(f64), s["rstd"][rows].to(f64).unsqueeze(1)
            xh = (s["x"][rows].to(f64) - s["mean"][rows].to(f64).unsqueeze(1)) * r
            dgamma += torch.einsum("nk,nk->k", dy, xh)
            dbeta += dy.sum(0)
            q = dy * s["gamma"].to(f64)
            dx[rows] = (q - q.mean(1, True) - xh * (q * xh).mean(1, True)) * r
        return dx, dgamma, dbeta
    if do == "loss":
        loss = torch.zeros(case["n"], dtype=f64, device=DEV)
        grad = torch.zeros(case["n"], case["m"], dtype=f64, device=DEV)
        for a, (lo, hi) in enumerate(zip(s["ends"], s["ends"][1:])):
            c = int(s["n_classes"][a])
            if lo == hi:
                continue
            logp = torch.log_softmax(s["logits"][lo:hi, :c].to(f64), 1)
            rows = torch.nonzero(s["label"][lo:hi] >= 0)[:, 0]
            at = s["label"][lo:hi][rows].long()
            w = torch.ones(hi - lo, dtype=f64, device=DEV) if not case["weighted"] else s["weight"][lo:hi].to(f64)
            loss[lo + rows] = -logp[rows, at] * w[rows]
            p = logp.exp()
            p[rows, at] -= 1.0
            keep = torch.zeros(hi - lo, dtype=f64, device=DEV)
            keep[rows] = w[rows] * s["scale"]
            grad[lo:hi, :c] = p * keep.unsqueeze(1)
        return loss, grad
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(v.to(f64)) for v in s["grads"]])).reshape(1)
    c = min(1.0, case["max_norm"] / (float(norm) + 1e-6))
    return norm, torch.cat(s["grads"]).to(f64).mul_(c)
