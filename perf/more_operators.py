"""What is measured of the operators for heads that are made of experts: routing, moving rows, dropout, products in 8 bits.

Such a head has many small networks, the experts, and a router: a linear layer whose outputs, one for every expert, say
which few of them a row goes through and with what weights.  Rows are brought together by expert, go through the grouped
linear layers, and come back as weighted sums.  `do` says which operator a case calls:

  route          each row's experts and their weights from the router's logits, and every (row, expert) pair's place
                 among the rows sorted by expert
  route_back     the gradient of the logits from that of the weights
  dispatch       rows copied to their places
  combine        weighted sums of the rows at their places, and a residual
  combine_back   its gradients with respect to the rows at their places and the weights
  dropout        elements set to zero by random numbers that are computed from a seed and the element's position
  linear8        a grouped linear layer for serving: rows rounded to 8 bits with a scale for each, weights in 8 bits with a
                 scale for each output
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
INF = float("inf")


def _case(name, **kw):
    c = dict(do="route", bf16=False, n=1, experts=1, top=1, sigmoid=False, bias=False, groups=1, top_groups=1, renormalize=True,
             scale=1.0, masked=0.0, d=1, dropped=0.0, weighted=True, residual=False, p=0.1, k=1, m=1, relu=False, skew=0.0, wide_out=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request that is served: latency is all that counts
        _case("route_one_request", n=1, experts=64, top=6, sigmoid=True, bias=True, groups=8, top_groups=4, scale=2.5),
        # a batch of a small model whose experts are not all there for every row
        _case("route_batch_bf16", bf16=True, n=4097, experts=60, top=4, renormalize=False, masked=0.05),
        # the largest batch over many experts in groups, with a bias that balances them
        _case("route_256k_f32", n=262144, experts=256, top=8, sigmoid=True, bias=True, groups=8, top_groups=4, scale=2.5),
        # a training step's gradient of the router: softmax over all experts
        _case("route_back_64k_bf16", do="route_back", bf16=True, n=65536, experts=128, top=8, renormalize=False),
        # hidden rows on their way to the experts
        _case("dispatch_64k_bf16", do="dispatch", bf16=True, n=65536, d=512, experts=64, top=4),
        # a small model's way back, with the residual
        _case("combine_64k_f32", do="combine", n=65536, d=256, experts=16, top=2, residual=True),
        # a training step: many experts, some pairs dropped because their expert was full
        _case("combine_back_32k_bf16", do="combine_back", bf16=True, n=32768, d=768, experts=128, top=8, dropped=0.05),
        # a hidden layer of a small batch, of an odd width
        _case("dropout_small_f32", do="dropout", n=100, d=129, p=0.5),
        # hidden rows of a training step, added to the residual
        _case("dropout_64k_bf16", do="dropout", bf16=True, n=65536, d=768, residual=True),
        # one request through a hidden layer of one of eight applications
        _case("linear8_one_request", do="linear8", bf16=True, n=1, experts=8, k=512, m=256, relu=True),
        # logits of a window's queue: widths that no tile divides, float32 results
        _case("linear8_odd", do="linear8", bf16=True, n=10007, experts=12, skew=1.0, k=770, m=515, wide_out=True),
        # the largest batch through a hidden layer of sixteen experts
        _case("linear8_256k", do="linear8", bf16=True, n=262144, experts=16, skew=0.5, k=1024, m=1024, relu=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw(rng):
    do = rng.choice(["route", "route", "route", "route_back", "dispatch", "combine", "combine_back", "dropout", "dropout", "linear8", "linear8",
                     "linear8"])
    bf16 = rng.random() < 0.5
    # half of the sizes are multiples of 8 or 32, as configurations have them, the others are any number
    experts = _log_int(rng, 1, 32) * 8 if rng.random() < 0.5 else _log_int(rng, 2, 256)
    top = min(experts, _log_int(rng, 1, 8))
    if do in ("route", "route_back"):
        c = dict(do=do, bf16=bf16, n=_log_int(rng, 1, 262144), experts=experts, top=top, sigmoid=rng.random() < 0.5,
                 renormalize=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]), masked=rng.choice([0.0, 0.0, 0.05]))
        if do == "route":
            c["bias"] = rng.random() < 0.5
            groups = rng.choice([1, 1, 2, 4, 8])
            if experts % groups == 0:
                least = -(-top * groups // experts)
                c.update(groups=groups, top_groups=rng.randint(least, groups))
        elif top == 1:
            c["renormalize"] = False                           # (a single weight of 1 has no gradient)
        return c
    if do in ("dispatch", "combine", "combine_back"):
        d = _log_int(rng, 1, 64) * 32 if rng.random() < 0.5 else _log_int(rng, 3, 2048)
        return dict(do=do, bf16=bf16, n=_log_int(rng, 1, 131072), d=d, experts=experts, top=top, dropped=rng.choice([0.0, 0.05]),
                    weighted=do == "combine_back" or rng.random() < 0.7, residual=do == "combine" and rng.random() < 0.5)
    if do == "dropout":
        d = _log_int(rng, 1, 64) * 32 if rng.random() < 0.5 else _log_int(rng, 3, 4096)
        return dict(do=do, bf16=bf16, n=_log_int(rng, 1, 1048576), d=d, p=rng.choice([0.1, 0.25, 0.5]), residual=rng.random() < 0.5)
    k, m = ((_log_int(rng, 1, 32) * 32) if rng.random() < 0.5 else _log_int(rng, 3, 1024) for _ in range(2))
    return dict(do=do, bf16=bf16, n=_log_int(rng, 1, 262144), experts=_log_int(rng, 1, 32), skew=rng.choice([0.0, 0.5, 1.0]), k=k, m=m,
                relu=rng.random() < 0.5, wide_out=bf16 and rng.random() < 0.3, residual=rng.random() < 0.3)


def draw(rng):
    most = [work(c) for c in listed()]
    bytes_, flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        c = _case(None, **_draw(rng))
        w = work(c)
        if w["bytes"] <= bytes_ and w["flops"] <= flops:
            return c


def _sizes(n, groups, skew):
    """Rows of each group: shares proportional to (g + 1)^-skew, remainders to the first ones."""
    share = [(g + 1.0) ** -skew for g in range(groups)]
    out = [int(n * s / sum(share)) for s in share]
    for i in range(n - sum(out)):
        out[i % groups] += 1
    return out


def work(case):
    do, n, d, top, k, m = case["do"], case["n"], case["d"], case["top"], case["k"], case["m"]
    e = 2 if case["bf16"] else 4
    if do == "route":
        out = 12 * n * top + 4 * (case["experts"] + 1)          # experts, weights, places; offsets
        return {"bytes": n * case["experts"] * e + out, "flops": 8 * n * case["experts"]}
    if do == "route_back":
        # softmax over all experts needs every logit, the others only the chosen ones'
        read = n * case["experts"] * e if not case["sigmoid"] and not case["renormalize"] else n * top * e
        return {"bytes": read + n * case["experts"] * e + 8 * n * top, "flops": 6 * n * case["experts"]}
    if do in ("dispatch", "combine", "combine_back"):
        pairs = round(n * top * (1.0 - case["dropped"]))
        at = 4 * n * top
        if do == "dispatch":
            return {"bytes": (n + pairs) * d * e + at, "flops": 0}
        w = at if case["weighted"] else 0
        if do == "combine":
            return {"bytes": (n * (2 if case["residual"] else 1) + pairs) * d * e + at + w, "flops": 2 * pairs * d}
        return {"bytes": (n + 2 * pairs) * d * e + at + 2 * w, "flops": 3 * pairs * d}
    if do == "dropout":
        return {"bytes": n * d * e * (3 if case["residual"] else 2), "flops": 2 * n * d}
    held = sum(1 for s in _sizes(n, case["experts"], case["skew"]) if s)
    out = 4 if case["wide_out"] else e
    b = n * k * e + held * (k * m + 8 * m) + n * m * out * (2 if case["residual"] else 1) + 4 * (case["experts"] + 1)
    return {"bytes": b, "flops": 2 * n * k * m}


def _places(expert, experts):
    """Each pair's place among the pairs sorted by expert, in their order; -1 for pairs without an expert."""
    flat = expert.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    ordered, perm = torch.sort(key, stable=True)
    place = torch.empty_like(perm)
    place[perm] = torch.arange(perm.numel(), device=DEV)
    offsets = torch.searchsorted(ordered, torch.arange(experts + 1, device=DEV))
    return offsets.int(), torch.where(flat < 0, -1, place).int().view_as(expert)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    do, n, d, top, experts, k, m = (case[v] for v in ("do", "n", "d", "top", "experts", "k", "m"))
    t = torch.bfloat16 if case["bf16"] else torch.float32

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, device=DEV, generator=g) * scale).to(dtype)

    def room(*shape, dtype=t):
        return torch.zeros(*shape, dtype=dtype, device=DEV)

    s = dict(case=case)
    if do in ("route", "route_back"):
        s["logits"] = normal(n, experts, scale=1.5)
        if case["masked"]:
            # experts that are not there for a row, and rows that have none at all
            hide = torch.rand(n, experts, device=DEV, generator=g) < case["masked"]
            hide |= torch.rand(n, 1, device=DEV, generator=g) < 0.01
            s["logits"].masked_fill_(hide, -INF)
        if do == "route":
            s["bias"] = normal(experts, scale=0.1, dtype=torch.float32) if case["bias"] else None
            s["expert"], s["weight"] = room(n, top, dtype=torch.int32), room(n, top, dtype=torch.float32)
            s["offsets"], s["place"] = room(experts + 1, dtype=torch.int32), room(n, top, dtype=torch.int32)
        else:
            value, at = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
            s["expert"] = torch.where(value[:, :top] > -INF, at[:, :top], -1).int().contiguous()
            s["dweight"] = normal(n, top, dtype=torch.float32)
            s["dlogits"] = room(n, experts)
    elif do in ("dispatch", "combine", "combine_back"):
        # some experts are chosen more often than others
        lean = normal(1, experts, scale=0.5, dtype=torch.float32)
        expert = torch.sort(lean + normal(n, experts, dtype=torch.float32), dim=1, descending=True).indices[:, :top]
        if case["dropped"]:
            expert = torch.where(torch.rand(n, top, device=DEV, generator=g) < case["dropped"], -1, expert)
        s["place"] = _places(expert, experts)[1]
        s["weight"] = torch.rand(n, top, device=DEV, generator=g) if case["weighted"] else None
        if do == "dispatch":
            s["x"], s["xs"] = normal(n, d), room(n * top, d)
        else:
            s["ys"] = normal(n * top, d)
            if do == "combine":
                s["r"], s["y"] = normal(n, d) if case["residual"] else None, room(n, d)
            else:
                s["dy"], s["dys"], s["dweight"] = normal(n, d), room(n * top, d), room(n, top, dtype=torch.float32)
    elif do == "dropout":
        s["x"], s["r"], s["y"] = normal(n, d), normal(n, d) if case["residual"] else None, room(n, d)
        s["seed"], s["offset"] = 0x5DEECE66D ^ (seed * 0x9E3779B97F4A7C15 & (1 << 63) - 1), 1000003 * (seed % 1000)
    else:
        sizes = _sizes(n, experts, case["skew"])
        turn = seed % experts                  # which expert has the most rows changes with the seed
        sizes = sizes[turn:] + sizes[:turn]
        ends = [0]
        for v in sizes:
            ends.append(ends[-1] + v)
        s["ends"], s["offsets"] = ends, torch.tensor(ends, dtype=torch.int32, device=DEV)
        s["x"] = normal(n, k)
        # the weights as a program that serves keeps them: whole numbers and their scales, an output's inputs next to each other
        w = normal(experts, m, k, scale=math.sqrt(2.0 / k), dtype=torch.float32)
        s["w_scale"] = w.abs().amax(2) / 127.0
        s["w"] = torch.round(w / s["w_scale"][:, :, None]).to(torch.int8)
        s["b"] = normal(experts, m, scale=0.1, dtype=torch.float32)
        s["out"] = torch.float32 if case["wide_out"] else t
        s["r"] = normal(n, m, dtype=s["out"]) if case["residual"] else None
        s["q"], s["q_scale"] = room(n, k, dtype=torch.int8), room(n, dtype=torch.float32)
        s["y"] = room(n, m, dtype=s["out"])
    if own:
        from paper_2505_06641_amd import binding
        s["ops"] = binding.Ops()
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    ops, case, do = s["ops"], s["case"], s["case"]["do"]
    if do == "route":
        ops.sp_route(s["logits"], s["expert"], s["weight"], sigmoid=case["sigmoid"], bias=s["bias"], groups=case["groups"],
                     top_groups=case["top_groups"], renormalize=case["renormalize"], scale=case["scale"])
        ops.sp_route_order(s["expert"], s["offsets"], s["place"])
        return s["expert"], s["weight"], s["offsets"], s["place"]
    if do == "route_back":
        ops.sp_route_backward(s["logits"], s["expert"], s["dweight"], s["dlogits"], sigmoid=case["sigmoid"],
                              renormalize=case["renormalize"], scale=case["scale"])
        return s["dlogits"]
    if do == "dispatch":
        ops.sp_dispatch(s["x"], s["place"], s["xs"])
        return s["xs"]
    if do == "combine":
        ops.sp_combine(s["ys"], s["place"], s["y"], weight=s["weight"], residual=s["r"])
        return s["y"]
    if do == "combine_back":
        ops.sp_combine_backward(s["dy"], s["ys"], s["place"], s["weight"], dys=s["dys"], dweight=s["dweight"])
        return s["dys"], s["dweight"]
    if do == "dropout":
        ops.sp_dropout(s["x"], s["y"], case["p"], s["seed"], offset=s["offset"], residual=s["r"])
        return s["y"]
    ops.sp_quantize_rows(s["x"], s["q"], s["q_scale"])
    ops.sp_grouped_linear_quantized(s["q"], s["q_scale"], s["offsets"], s["w"], s["w_scale"], s["y"], bias=s["b"], relu=case["relu"],
                                    residual=s["r"])
    return s["y"]


def _philox(c0, c1, c2, c3, k0, k1):
    """Ten rounds of Philox 4x32 (Salmon, Moraes, Dror and Shaw, 2011) on 32-bit words that are held in 64 bits."""
    low = 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # (the low 64 bits are right whatever the sign)
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _plain(s):
    case, do = s["case"], s["case"]["do"]
    n, d, top, experts = case["n"], case["d"], case["top"], case["experts"]
    if do == "route":
        z = s["logits"].float()
        there = z > -INF
        if s["bias"] is not None or case["groups"] > 1:
            # which experts are chosen hangs on small differences: in 64 bits
            zd = z.double()
            if case["sigmoid"]:
                c = 1.0 / (1.0 + torch.exp(-zd))
            else:
                e = torch.exp(zd - torch.where(there, zd, -1e300).max(1, keepdim=True).values)
                c = e / e.sum(1, keepdim=True)
            if s["bias"] is not None:
                c = c + s["bias"].double()
        else:
            c = z
        c = torch.where(there, c, -INF)
        if case["groups"] > 1:
            by = c.view(n, case["groups"], experts // case["groups"])
            best = torch.sort(by, dim=2, descending=True).values[:, :, :2]
            value = torch.where(best > -INF, best, 0.0).sum(2)
            value = torch.where(best[:, :, 0] > -INF, value, -INF)
            kept = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
            keep = torch.zeros_like(value, dtype=torch.bool).scatter(1, kept, True)
            c = torch.where(keep[:, :, None], by, -INF).view(n, experts)
        value, at = torch.sort(c, dim=1, descending=True, stable=True)
        value, at = value[:, :top], at[:, :top]
        chosen = value > -INF
        zc = z.gather(1, at)
        if case["sigmoid"]:
            w = torch.where(chosen, 1.0 / (1.0 + torch.exp(-zc)), 0.0)
        else:
            over = zc if case["renormalize"] else z
            w = torch.where(chosen, torch.exp(zc - over.max(1, keepdim=True).values), 0.0)
            if not case["renormalize"]:
                w = w / torch.exp(z - z.max(1, keepdim=True).values).sum(1, keepdim=True)
        if case["renormalize"]:
            w = w / w.sum(1, keepdim=True)
        w = torch.where(chosen, w * case["scale"], 0.0)
        expert = torch.where(chosen, at, -1).int()
        return (expert, w) + _places(expert, experts)
    if do == "route_back":
        z = s["logits"].float()
        chosen = s["expert"] >= 0
        at = s["expert"].clamp(min=0).long()
        zc = z.gather(1, at)
        dw = torch.where(chosen, s["dweight"], 0.0) * case["scale"]
        if case["sigmoid"]:
            sc = torch.where(chosen, 1.0 / (1.0 + torch.exp(-zc)), 0.0)
            dz = dw * sc
            if case["renormalize"]:
                w = sc / sc.sum(1, keepdim=True)
                dz = w * (dw - (dw * w).sum(1, keepdim=True))
            dz = dz * (1.0 - sc)
        elif case["renormalize"]:
            w = torch.where(chosen, torch.exp(zc - zc.max(1, keepdim=True).values), 0.0)
            w = w / w.sum(1, keepdim=True)
            dz = w * (dw - (dw * w).sum(1, keepdim=True))
        else:
            e = torch.exp(z - z.max(1, keepdim=True).values)
            e = torch.where(z > -INF, e / e.sum(1, keepdim=True), 0.0)
            sc = e.gather(1, at)
            dz = dw * sc
            return (-e * dz.sum(1, keepdim=True)).scatter_add(1, at, torch.where(chosen, dz, 0.0)).to(s["logits"].dtype)
        return torch.zeros_like(z).scatter_add(1, at, torch.where(chosen, dz, 0.0)).to(s["logits"].dtype)
    if do in ("dispatch", "combine", "combine_back"):
        here = s["place"] >= 0
        at = s["place"].clamp(min=0).long()
        if do == "dispatch":
            s["xs"][at[here]] = s["x"][:, None, :].expand(n, top, d)[here]
            return s["xs"]
        rows = torch.where(here[:, :, None], s["ys"][at].float(), 0.0)
        if do == "combine":
            y = (rows if s["weight"] is None else rows * s["weight"][:, :, None]).sum(1)
            return (y if s["r"] is None else y + s["r"].float()).to(s["y"].dtype)
        dy = s["dy"].float()[:, None, :]
        s["dys"][at[here]] = (dy * s["weight"][:, :, None])[here].to(s["dys"].dtype)
        return s["dys"], (rows * dy).sum(2)
    if do == "dropout":
        drop = round(case["p"] * 65536)
        # eight elements of a row share a counter: the piece of the row, the row, and the offset; 16 bits for each element
        piece = torch.arange((d + 7) // 8, device=DEV).expand(n, -1)
        row = torch.arange(n, device=DEV)[:, None].expand_as(piece)
        off, key = s["offset"], s["seed"]
        words = torch.stack(_philox(piece, row, torch.full_like(piece, off & 0xFFFFFFFF), torch.full_like(piece, off >> 32), key & 0xFFFFFFFF,
                                    key >> 32), 2)
        bits = torch.stack([words & 0xFFFF, words >> 16], 3).view(n, -1)[:, :d]
        y = torch.where(bits >= drop, s["x"].float() * (65536.0 / (65536 - drop)), 0.0)
        return (y if s["r"] is None else y + s["r"].float()).to(s["y"].dtype)
    x = s["x"].float()
    top_x = x.abs().amax(1, keepdim=True)
    most = torch.full_like(top_x, 127.0)                          # (one rounding: a number over a tensor is a product with its inverse)
    q, scale = torch.round(x * (most / top_x)), top_x / most
    y = torch.empty_like(s["y"])
    for a in range(experts):
        lo, hi = s["ends"][a], s["ends"][a + 1]
        if lo == hi:
            continue
        z = (q[lo:hi] @ s["w"][a].float().t()) * scale[lo:hi] * s["w_scale"][a] + s["b"][a]
        if case["relu"]:
            z = torch.where(z < 0, 0.0, z)
        y[lo:hi] = z if s["r"] is None else z + s["r"][lo:hi].float()
    return y


def _exact_philox(counter, key):
    """The same numbers, whole arrays of unsigned words at a time on the host."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    mul, add, k = (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57)), (0x9E3779B9, 0xBB67AE85), list(key)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = mul[0] * c[0], mul[1] * c[2]
        c = [(q >> half) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> half) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[i] + add[i]) % (1 << 32) for i in range(2)]
    return c


def exact(case, seed):
    """The operators' values in 64 bits, from their definitions."""
    s = prepare(case, seed)
    do, f64 = case["do"], torch.float64
    n, d, top, experts = case["n"], case["d"], case["top"], case["experts"]
    if do == "route":
        z = s["logits"].to(f64)
        score = torch.sigmoid(z) if case["sigmoid"] else torch.softmax(z, 1).nan_to_num(0.0)
        value = score if s["bias"] is None else score + s["bias"].to(f64)
        if s["bias"] is None and case["groups"] == 1:
            value = z.clone()
        value[z == -INF] = -INF
        if case["groups"] > 1:
            width = experts // case["groups"]
            pair = torch.topk(value.view(n, -1, width), min(2, width), dim=2).values
            total = pair.masked_fill(pair == -INF, 0.0).sum(2).masked_fill(pair[:, :, 0] == -INF, -INF)
            closed = torch.ones(n, case["groups"], dtype=torch.bool, device=DEV)
            for _ in range(case["top_groups"]):
                closed.scatter_(1, (total == total.amax(1, True)).int().argmax(1, True), False)
                total.masked_fill_(~closed, -INF)
            value.view(n, -1, width).masked_fill_(closed[:, :, None], -INF)
        expert = torch.full((n, top), -1, dtype=torch.int64, device=DEV)
        for j in range(top):
            high = value.amax(1, True)
            at = (value == high).int().argmax(1, True)
            expert[:, j:j + 1] = torch.where(high > -INF, at, -1)
            value.scatter_(1, at, -INF)
        got = expert >= 0
        at = expert.clamp(min=0)
        if case["renormalize"]:
            part = torch.nn.functional.logsigmoid(z.gather(1, at)) if case["sigmoid"] else z.gather(1, at)
            w = torch.softmax(part.masked_fill(~got, -INF), 1).nan_to_num(0.0)
        else:
            w = score.gather(1, at) * got
        flat = expert.reshape(-1)
        counts = torch.zeros(experts + 1, dtype=torch.int64, device=DEV)
        counts.scatter_add_(0, flat + 1, torch.ones_like(flat))
        offsets = torch.cumsum(counts, 0) - counts[0]
        place = torch.empty_like(flat)
        place[torch.argsort(flat, stable=True)] = torch.arange(flat.numel(), device=DEV) - counts[0]
        place = place.view(n, top).masked_fill(~got, -1)
        return expert.int(), w * case["scale"], offsets.int(), place.int()
    if do == "route_back":
        # the derivative along each weight, summed over the chosen ones
        z = s["logits"].to(f64)
        got = (s["expert"] >= 0).to(f64)
        at = s["expert"].clamp(min=0).long()
        dw = s["dweight"].to(f64) * got * case["scale"]
        hit = torch.zeros_like(z).scatter_add_(1, at, got)
        up = torch.zeros_like(z).scatter_add_(1, at, dw)
        score = torch.sigmoid(z) if case["sigmoid"] else torch.softmax(z, 1).nan_to_num(0.0)
        if case["renormalize"]:
            total = (score * hit).sum(1, True)
            up = hit * (up - (up * score).sum(1, True) / total) / total
            up.nan_to_num_(0.0)
        if case["sigmoid"]:
            return up * score * (1.0 - score)
        return score * (up - (up * score).sum(1, True))
    if do in ("dispatch", "combine", "combine_back"):
        place = s["place"].long()
        if do == "dispatch":
            out = torch.zeros(n * top, d, dtype=f64, device=DEV)
            for j in range(top):
                rows = torch.nonzero(place[:, j] >= 0)[:, 0]
                out[place[rows, j]] = s["x"][rows].to(f64)
            return out
        if do == "combine":
            out = torch.zeros(n, d, dtype=f64, device=DEV) if s["r"] is None else s["r"].to(f64)
            for j in range(top):
                rows = torch.nonzero(place[:, j] >= 0)[:, 0]
                part = s["ys"][place[rows, j]].to(f64)
                if s["weight"] is not None:
                    part *= s["weight"][rows, j, None].to(f64)
                out.index_add_(0, rows, part)
            return out
        dys = torch.zeros(n * top, d, dtype=f64, device=DEV)
        dweight = torch.zeros(n, top, dtype=f64, device=DEV)
        for j in range(top):
            rows = torch.nonzero(place[:, j] >= 0)[:, 0]
            up = s["dy"][rows].to(f64)
            dys[place[rows, j]] = up * s["weight"][rows, j, None].to(f64)
            dweight[rows, j] = (up * s["ys"][place[rows, j]].to(f64)).sum(1)
        return dys, dweight
    if do == "dropout":
        if n * d > 1 << 27:
            return None
        off, key, wide = s["offset"], s["seed"], (d + 7) // 8
        at = np.arange(n * wide, dtype=np.uint64)
        full = np.full_like(at, off & 0xFFFFFFFF), np.full_like(at, off >> 32)
        words = _exact_philox((at % np.uint64(wide), at // np.uint64(wide)) + full, (key & 0xFFFFFFFF, key >> 32))
        words = np.stack(words, 1).astype(np.uint32)
        bits = words.view(np.uint16).reshape(n, wide * 8)[:, :d]              # low half first
        drop = int(math.floor(case["p"] * 65536 + 0.5))
        kept = torch.from_numpy(np.ascontiguousarray(bits >= drop)).to(DEV)
        y = s["x"].to(f64) * kept / (1.0 - drop / 65536.0)
        return y if s["r"] is None else y + s["r"].to(f64)
    out = torch.empty(n, case["m"], dtype=f64, device=DEV)
    x = s["x"].float()
    high = x.abs().amax(1, keepdim=True)
    by = torch.div(torch.full_like(high, 127.0), high)
    q, scale = torch.round(x * by).to(f64), high.to(f64) / 127.0      # what the rows stand for is the operator's definition
    w = s["w"].to(f64) * s["w_scale"].to(f64)[:, :, None]
    for a, (lo, hi) in enumerate(zip(s["ends"], s["ends"][1:])):
        z = torch.addmm(s["b"][a].to(f64), q[lo:hi] * scale[lo:hi], w[a].t())
        if case["relu"]:
            z.clamp_(min=0)
        out[lo:hi] = z if s["r"] is None else z + s["r"][lo:hi].to(f64)
    return out
