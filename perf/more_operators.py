"""The operators of layers in 8-bit floating point and of sparse feed-forward layers, as they are measured.

Five kinds of cases, each one pass of what a training or serving program does:

linear   Y = X W^T, both operands in 8-bit floating point (a sign, four exponent and three mantissa bits, largest value 448), a power-of-two
         scale for every block of 128 along the summed axis; a tile of 128 x 128 of the weights shares one.  W laid out once,
         X quantized in the call.
train    the same layer's forward pass and both gradients: dX = dY W, dW = dY^T X, the latter in blocks of 128 tokens; all of the type of X.
route    a router: softmax or sigmoid scores of the logits, a bias that counts for the choice only, groups of experts of which the best
         (by the sum of their two best) stay, the k best experts, their scores as weights, renormalised or not; the order of the rows
         by expert; with "train" the gradient of the logits.
experts  every expert's rows through its own weights, in the same 8 bits, rows ordered by expert; with "train" the gradients of the
         rows and of all weights.
combine  the weighted sum of a token's rows; with "train" its gradients.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 128


def listed():
    return [
        # serving: one token through an expanding layer
        {"name": "linear_one_token", "kind": "linear", "M": 1, "N": 8192, "K": 4096, "dtype": "bf16", "out": "bf16"},
        # serving: a few requests at once, odd sizes, fp32 in and out
        {"name": "linear_few_tokens", "kind": "linear", "M": 21, "N": 2300, "K": 5130, "dtype": "fp32", "out": "fp32"},
        # a long prompt through a wide layer
        {"name": "linear_large", "kind": "linear", "M": 16384, "N": 8192, "K": 8192, "dtype": "bf16", "out": "bf16"},
        # a training step of a small layer on a ragged batch
        {"name": "train_ragged", "kind": "train", "M": 1111, "N": 1500, "K": 2030, "dtype": "fp32"},
        # a training step of a wide layer
        {"name": "train_large", "kind": "train", "M": 8192, "N": 8192, "K": 4096, "dtype": "bf16"},
        # serving: the router of a few requests
        {"name": "route_few_tokens", "kind": "route", "T": 5, "E": 60, "k": 4, "scores": "softmax", "bias": False, "groups": 1, "top_groups": 1,
         "renormalize": False, "scale": 1.0, "dtype": "bf16", "train": False, "padded": 0},
        # training: the router of a large batch with many experts in groups
        {"name": "route_large", "kind": "route", "T": 16384, "E": 256, "k": 8, "scores": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "renormalize": True, "scale": 2.5, "dtype": "fp32", "train": True, "padded": 77},
        # serving: a few tokens, each with its own experts
        {"name": "experts_few_tokens", "kind": "experts", "T": 4, "k": 6, "E": 64, "N": 2816, "K": 2048, "dtype": "bf16", "train": False},
        # training on a ragged batch, experts of a few dozen to some hundreds of rows, odd in every size
        {"name": "experts_ragged", "kind": "experts", "T": 1001, "k": 2, "E": 12, "N": 1100, "K": 777, "dtype": "fp32", "train": True},
        # training on a large batch
        {"name": "experts_large", "kind": "experts", "T": 16384, "k": 4, "E": 32, "N": 2048, "K": 2048, "dtype": "bf16", "train": True},
        # serving: the sum of a few tokens' rows
        {"name": "combine_few_tokens", "kind": "combine", "T": 3, "k": 8, "E": 64, "D": 5121, "dtype": "bf16", "train": False},
        # training: a large batch
        {"name": "combine_large", "kind": "combine", "T": 16384, "k": 4, "E": 32, "D": 4096, "dtype": "bf16", "train": True},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and n >= 128:
            n = n // 64 * 64
        return max(lo, min(hi, n))

    kind = rng.choice(["linear", "linear", "train", "route", "experts", "experts", "combine"])
    dtype = rng.choice(["bf16", "fp32"])
    if kind == "linear":
        return {"kind": kind, "M": size(1, 16384), "N": size(64, 8192), "K": size(64, 8192), "dtype": dtype, "out": rng.choice(["bf16", "fp32"])}
    if kind == "train":
        return {"kind": kind, "M": size(1, 8192), "N": size(64, 8192), "K": size(64, 4096), "dtype": dtype}
    T, train = size(1, 16384), rng.random() < 0.5
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        per = rng.randint(2, 256 // groups)
        top = rng.randint(1, groups)
        return {"kind": kind, "T": T, "E": groups * per, "k": rng.randint(1, min(16, top * per)), "scores": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "top_groups": top, "renormalize": rng.random() < 0.6, "scale": rng.choice([1.0, 2.5]),
                "dtype": dtype, "train": train, "padded": T // 16 if rng.random() < 0.5 else 0}
    E = size(2, 64)
    k = rng.randint(1, min(8, E))
    if kind == "combine":
        return {"kind": kind, "T": T, "k": min(k, 4) if T > 8192 else k, "E": E, "D": size(64, 4096), "dtype": dtype, "train": train}
    T = max(1, min(T, 32768 // k))
    return {"kind": kind, "T": T, "k": k, "E": E, "N": size(64, 2048), "K": size(64, 2048), "dtype": dtype, "train": train}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activation(g, rows, cols, dtype):
    """Bell-shaped, with a few columns of much larger values, as hidden states have them."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    loud = torch.rand(cols, generator=g, device="cuda") < 0.005
    return (x * (1 + 19 * loud)).to(DT[dtype])


def _gradient(g, rows, cols, dtype):
    """Sharp, with long tails, and a spread of its own in every column."""
    u = torch.rand(rows, cols, generator=g, device="cuda") - 0.5
    spread = 10 ** (-2 * torch.rand(cols, generator=g, device="cuda") - 1)
    return (-torch.sign(u) * torch.log1p(-2 * u.abs()).clamp_min(-16) * spread).to(DT[dtype])


def _weight(g, E, N, K):
    return (torch.randn(E, N, K, generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)


def _choices(g, T, k, E):
    """k different experts for every token, some experts far more often than others."""
    popular = torch.randn(E, generator=g, device="cuda")
    return torch.topk(torch.randn(T, E, generator=g, device="cuda") + 0.7 * popular, k, dim=1).indices.to(torch.int32)


def _inputs(case, seed):
    g, k = _generator(seed), case["kind"]
    if k == "linear":
        return {"x": _activation(g, case["M"], case["K"], case["dtype"]), "w": _weight(g, 1, case["N"], case["K"])}
    if k == "train":
        return {"x": _activation(g, case["M"], case["K"], case["dtype"]), "w": _weight(g, 1, case["N"], case["K"]),
                "dy": _gradient(g, case["M"], case["N"], case["dtype"])}
    if k == "route":
        T, E = case["T"], case["E"]
        logits = (1.5 * torch.randn(T, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")).to(DT[case["dtype"]])
        if case["padded"]:
            logits[T - case["padded"]:] = -math.inf
        i = {"logits": logits, "dw": torch.randn(T, case["k"], generator=g, device="cuda")}
        i["bias"] = 0.05 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        return i
    chosen = _choices(g, case["T"], case["k"], case["E"])
    rows = case["T"] * case["k"]
    if k == "experts":
        return {"chosen": chosen, "x": _activation(g, case["T"], case["K"], case["dtype"]), "w": _weight(g, case["E"], case["N"], case["K"]),
                "dy": _gradient(g, rows, case["N"], case["dtype"]) if case["train"] else None}
    weights = torch.softmax(torch.randn(case["T"], case["k"], generator=g, device="cuda"), 1)
    return {"chosen": chosen, "y": _activation(g, rows, case["D"], case["dtype"]), "weights": weights,
            "dout": _gradient(g, case["T"], case["D"], case["dtype"]) if case["train"] else None}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    k = case["kind"]
    if own:
        from paper_2102_04782_amd import binding as daq

        s["daq"] = daq
        if k in ("linear", "train", "experts"):      # laid out once, as a program keeps its weights
            s["w"], s["w_t"] = daq.fp8_quantize_weights(s["w"])
        if k == "route":
            s["scores"] = {"softmax": daq.SCORES_SOFTMAX, "sigmoid": daq.SCORES_SIGMOID}[case["scores"]]
        if k in ("experts", "combine"):              # what the router has handed on
            s["plan"] = daq.experts_plan(s["chosen"], case["E"])
    else:
        if k in ("linear", "train", "experts"):
            s["w"] = _weight_values(s["w"])
        if k in ("experts", "combine"):
            s["order"], s["place"], s["counts"] = _order(s["chosen"], case["E"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _power(e):
    """2^e of whole numbers -126 .. 127, in 32 bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _values(b, top):
    """The 8-bit values of b, 32 bits, with one scale for what shares the largest magnitude `top`."""
    bits = top.view(torch.int32)
    e = ((bits >> 23).long() - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).long()).clamp_min(-126)
    t = b.abs() * _power(-e)
    step = _power(((t.view(torch.int32) >> 23).long() - 127).clamp_min(-6) - 3)
    v = torch.round(t / step) * step
    return torch.where(b < 0, -v, v) * _power(e)


def _row_values(x):
    """Blocks of 128 along the rows of x."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).reshape(rows, -1, BLOCK)
    return _values(b, b.abs().amax(2, keepdim=True)).view(rows, -1)[:, :cols]


def _weight_values(w):
    """Tiles of 128 x 128 of every matrix of w [E, N, K]."""
    E, N, K = w.shape
    b = torch.nn.functional.pad(w.float(), (0, -K % BLOCK, 0, -N % BLOCK))
    b = b.reshape(E, -(-N // BLOCK), BLOCK, -(-K // BLOCK), BLOCK)
    return _values(b, b.abs().amax((2, 4), keepdim=True)).view(E, -(-N // BLOCK) * BLOCK, -1)[:, :N, :K].contiguous()


def _order(chosen, E):
    """Slots (token * k + j) by expert, in their order within one, -1 behind the last; the place of every slot; rows of every expert."""
    flat = chosen.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    counts = torch.bincount(key, minlength=E + 1)[:E]
    order = torch.where(torch.arange(order.numel(), device=order.device) < counts.sum(), order, -1)
    return order.int(), torch.where(flat < 0, -1, place).int().view(chosen.shape), counts.int()


def _route_plain(s):
    case, T, E, k = s["case"], s["case"]["T"], s["case"]["E"], s["case"]["k"]
    x = s["logits"].double()                 # scores next to one another have to be told apart
    there = x > -math.inf
    if case["scores"] == "softmax":
        e = torch.where(there, torch.exp(x - x.amax(1, keepdim=True).clamp_min(-1e300)), 0.0)
        score = e / e.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        score = torch.where(there, 1 / (1 + torch.exp(-x)), 0.0)
    c = score if s["bias"] is None else score + s["bias"].double()
    c = torch.where(there, c, -math.inf)
    if case["groups"] > 1:
        by = c.view(T, case["groups"], -1)
        best = torch.sort(by, dim=2, descending=True).values[:, :, :2]
        total = torch.where(best > -math.inf, best, 0.0).sum(2)
        total = torch.where(best[:, :, 0] > -math.inf, total, -math.inf)
        first = torch.sort(total, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        stays = torch.zeros_like(total, dtype=torch.bool).scatter_(1, first, True)
        c = torch.where(stays.unsqueeze(2), by, -math.inf).view(T, E)
    top = torch.sort(c, dim=1, descending=True, stable=True)
    chosen = top.indices[:, :k]
    ok = top.values[:, :k] > -math.inf
    sc = torch.where(ok, score.gather(1, chosen), 0.0)
    total = sc.sum(1, keepdim=True) if case["renormalize"] else torch.ones_like(sc[:, :1])
    total = torch.where(total > 0, total, 1.0)
    w = sc / total * case["scale"]
    experts = torch.where(ok, chosen, -1).int()
    order, place, counts = _order(experts, E)
    out = {"weights": w.float(), "experts": experts, "order": order, "place": place, "counts": counts}
    if case["train"]:
        g = s["dw"].double()
        ds = case["scale"] * g
        if case["renormalize"]:
            ds = case["scale"] / total * (g - (g * sc).sum(1, keepdim=True) / total)
        ds = torch.zeros_like(score).scatter_add_(1, chosen, torch.where(ok, ds, 0.0))
        if case["scores"] == "sigmoid":
            d = ds * score * (1 - score)
        else:
            d = score * (ds - (ds * score).sum(1, keepdim=True))
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _experts_plain(s):
    case, to = s["case"], s["x"].dtype
    token = torch.div(s["order"].long(), case["k"], rounding_mode="floor")
    x = _row_values(s["x"])
    y = torch.empty(token.numel(), case["N"], device=x.device)
    train = case["train"]
    if train:
        d = _row_values(s["dy"])
        dx = torch.empty(token.numel(), case["K"], device=x.device)
        dw = torch.zeros(case["E"], case["N"], case["K"], device=x.device)
    at = 0
    for e, n in enumerate(s["counts"].tolist()):
        if n:
            here, w = slice(at, at + n), s["w"][e]
            y[here] = torch.matmul(x[token[here]], w.t())
            if train:
                dx[here] = torch.matmul(d[here], w)
                by_dy, by_x = _row_values(s["dy"][here].t()), _row_values(s["x"][token[here]].t())
                dw[e] = torch.matmul(by_dy, by_x.t())
        at += n
    return {"y": y.to(to), "dx": dx.to(to), "dw": dw.to(to)} if train else y.to(to)


def _combine_plain(s):
    case, to = s["case"], s["y"].dtype
    T, k, D = case["T"], case["k"], case["D"]
    place = s["place"].reshape(-1).long()
    y, w = s["y"].float()[place].view(T, k, D), s["weights"]
    out = (w.unsqueeze(2) * y).sum(1).to(to)
    if not case["train"]:
        return out
    d = s["dout"].float()
    dw = (d.unsqueeze(1) * y).sum(2)
    dy = torch.empty(T * k, D, dtype=to, device=d.device)
    dy[place] = (w.unsqueeze(2) * d.unsqueeze(1)).view(T * k, D).to(to)
    return {"out": out, "dy": dy, "dw": dw}


def _run_plain(s):
    case, k = s["case"], s["case"]["kind"]
    if k == "linear":
        return torch.matmul(_row_values(s["x"]), s["w"][0].t()).to(DT[case["out"]])
    if k == "train":
        x, dy, w = s["x"], s["dy"], s["w"][0]
        y, dx = torch.matmul(_row_values(x), w.t()), torch.matmul(_row_values(dy), w)
        dw = torch.matmul(_row_values(dy.t()), _row_values(x.t()).t())
        return {"y": y.to(x.dtype), "dx": dx.to(x.dtype), "dw": dw.to(x.dtype)}
    return {"route": _route_plain, "experts": _experts_plain, "combine": _combine_plain}[k](s)


def run(s):
    if not own:
        return _run_plain(s)
    daq, case, k = s["daq"], s["case"], s["case"]["kind"]
    if k == "linear":
        return daq.fp8_linear(s["x"], s["w"], dtype=DT[case["out"]])
    if k == "train":
        x, x_c = daq.fp8_quantize_both(s["x"])
        y = daq.fp8_matmul(x, s["w"], dtype=s["x"].dtype)
        dy, dy_c = daq.fp8_quantize_both(s["dy"])
        dx = daq.fp8_matmul(dy, s["w_t"], dtype=s["x"].dtype)
        return {"y": y, "dx": dx, "dw": daq.fp8_matmul(dy_c, x_c, dtype=s["x"].dtype)}
    if k == "route":
        form = {"scores": s["scores"], "renormalize": case["renormalize"], "scale": case["scale"]}
        weights, experts = daq.route(s["logits"], case["k"], bias=s["bias"], groups=case["groups"], top_groups=case["top_groups"], **form)
        plan = daq.experts_plan(experts, case["E"])
        out = {"weights": weights, "experts": experts, "order": plan.rows, "place": plan.place, "counts": plan.counts}
        if case["train"]:
            out["dlogits"] = daq.route_backward(s["dw"], s["logits"], experts, **form)
        return out
    plan = s["plan"]
    if k == "experts":
        if not case["train"]:
            return daq.experts_linear(s["x"], s["w"], plan)
        to = s["x"].dtype
        x, x_c = daq.experts_quantize(s["x"], plan)
        y = daq.experts_matmul(x, s["w"], plan, dtype=to)
        dy, dy_c = daq.experts_quantize(s["dy"], plan, sorted_rows=True)
        dx = daq.experts_matmul(dy, s["w_t"], plan, sorted_rows=True, dtype=to)
        return {"y": y, "dx": dx, "dw": daq.experts_weight_grad(dy_c, x_c, plan, dtype=to)}
    out = daq.experts_combine(s["y"], plan, s["weights"])
    if not case["train"]:
        return out
    dy, dw = daq.experts_combine_backward(s["dout"], s["y"], plan, s["weights"])
    return {"out": out, "dy": dy, "dw": dw}


def work(case):
    k = case["kind"]
    size = 2 if case["dtype"] == "bf16" else 4
    codes = lambda rows, cols: rows * cols + rows * -(-cols // BLOCK)
    if k == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": size * M * K + codes(N, K) + (2 if case["out"] == "bf16" else 4) * M * N, "flops": 2 * M * N * K}
    if k == "train":                     # x, dy and w; y, dx and dw
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * size * M * (K + N) + codes(N, K) + size * N * K, "flops": 6 * M * N * K}
    T, E, picks = case["T"], case["E"], case["T"] * case["k"]
    if k == "route":                     # logits in; weights, experts, order and place out; backwards logits, gradients and choices in, logits' gradients out
        n = size * T * E + 16 * picks + 4 * E
        return {"bytes": n + (2 * size * T * E + 8 * picks if case["train"] else 0), "flops": 20 * T * E}
    if k == "experts":                   # (weights of the experts that have rows)
        N, K, used = case["N"], case["K"], min(E, picks)
        n = size * T * K + codes(used * N, K) + size * picks * N
        if case["train"]:
            return {"bytes": n + size * picks * (N + K) + size * E * N * K, "flops": 6 * picks * N * K}
        return {"bytes": n, "flops": 2 * picks * N * K}
    D = case["D"]
    n = size * D * (picks + T) + 8 * picks
    return {"bytes": n + (size * D * (T + picks) + 4 * picks if case["train"] else 0), "flops": (6 if case["train"] else 2) * picks * D}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_round(v, largest):
    """v to the nearest multiple of a step, ties to even; largest: of what shares the scale, fp64."""
    frac, power = torch.frexp(largest)               # largest = frac * 2^power, frac in [.5, 1): 448 * 2^e = .875 * 2^(e + 9)
    e = torch.where(frac > 0.875, power - 8, power - 9).double()
    e = torch.where(largest > 0, e, torch.full_like(e, -126.0)).clamp(min=-126.0)
    t = v * torch.exp2(-e)
    low = (torch.frexp(t)[1].double() - 1).clamp(min=-6.0)
    low = torch.where(t == 0, torch.full_like(low, -6.0), low)
    unit = torch.exp2(low - 3)
    return torch.round(t / unit) * unit * torch.exp2(e)


def _exact_rows(x):
    """Blocks along rows, one column of blocks after the other."""
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        part = x[:, c:c + BLOCK]
        out[:, c:c + BLOCK] = _exact_round(part, part.abs().max(dim=1, keepdim=True).values)
    return out


def _exact_weight(w):
    w = w.double()
    out = torch.empty_like(w)
    for r in range(0, w.shape[0], BLOCK):
        for c in range(0, w.shape[1], BLOCK):
            part = w[r:r + BLOCK, c:c + BLOCK]
            out[r:r + BLOCK, c:c + BLOCK] = _exact_round(part, part.abs().max())
    return out


def _exact_columns(x):
    return _exact_rows(x.t().contiguous()).t().contiguous()


def _exact_plan(chosen, E):
    """Expert after expert."""
    flat = chosen.reshape(-1).cpu()
    order = torch.cat([torch.nonzero(flat == e)[:, 0] for e in range(E)])
    place = torch.full((flat.numel(),), -1, dtype=torch.int64)
    place[order] = torch.arange(order.numel())
    counts = torch.tensor([int((flat == e).sum()) for e in range(E)])
    order = torch.cat((order, torch.full((flat.numel() - order.numel(),), -1, dtype=torch.int64)))
    dev = chosen.device
    return order.int().to(dev), place.view(chosen.shape).int().to(dev), counts.int().to(dev)


def _exact_route(case, i):
    x, E, k = i["logits"].double(), case["E"], case["k"]
    empty = torch.isneginf(x)
    if case["scores"] == "softmax":
        score = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)
    else:
        score = torch.sigmoid(x)
    c = score if i["bias"] is None else score + i["bias"].double()
    c = c.masked_fill(empty, -math.inf)
    if case["groups"] > 1:
        per = E // case["groups"]
        best = c.view(-1, case["groups"], per).topk(min(2, per), dim=2).values
        total = best.clamp(min=-1e9).sum(2)          # (a row is empty as a whole or not at all)
        keep = torch.zeros_like(total, dtype=torch.bool)
        for _ in range(case["top_groups"]):
            keep.scatter_(1, _first_best(total.masked_fill(keep, -math.inf)), True)
        c = c.masked_fill(~keep.repeat_interleave(per, 1), -math.inf)
    left, chosen = c.clone(), []
    for _ in range(k):
        at = _first_best(left)
        chosen.append(torch.where(left.gather(1, at) > -math.inf, at, -1))
        left.scatter_(1, at, -math.inf)
    chosen = torch.cat(chosen, 1)
    mask = torch.zeros(x.shape[0], E + 1, dtype=torch.float64, device=x.device)
    mask.scatter_(1, torch.where(chosen < 0, E, chosen), 1.0)
    mask = mask[:, :E]
    total = (score * mask).sum(1, keepdim=True) if case["renormalize"] else torch.ones_like(x[:, :1])
    total = torch.where(total > 0, total, torch.ones_like(total))
    w = case["scale"] * score.gather(1, chosen.clamp(min=0)) * (chosen >= 0) / total
    order, place, counts = _exact_plan(chosen, E)
    out = {"weights": w, "experts": chosen.int(), "order": order, "place": place, "counts": counts}
    if case["train"]:
        # through the derivative of every score by every logit, summed over the chosen ones
        g = torch.zeros_like(x).scatter_add_(1, chosen.clamp(min=0), i["dw"].double() * (chosen >= 0))
        if case["renormalize"]:
            g = (g - (g * score * mask).sum(1, keepdim=True) / total) * mask
        g = g * case["scale"] / total
        out["dlogits"] = g * score * (1 - score) if case["scores"] == "sigmoid" else g * score - score * (g * score).sum(1, keepdim=True)
    return out


def _first_best(c):
    """[rows, 1]: the first of the largest."""
    top = c.max(dim=1, keepdim=True).values
    n = torch.arange(c.shape[1], device=c.device)
    return torch.where(c == top, n, c.shape[1]).min(dim=1, keepdim=True).values


def exact(case, seed):
    i, k = _inputs(case, seed), case["kind"]
    if k == "linear":
        return torch.mm(_exact_rows(i["x"]), _exact_weight(i["w"][0]).t().contiguous())
    if k == "train":
        w = _exact_weight(i["w"][0])
        return {"y": torch.mm(_exact_rows(i["x"]), w.t().contiguous()), "dx": torch.mm(_exact_rows(i["dy"]), w),
                "dw": torch.mm(_exact_columns(i["dy"]).t().contiguous(), _exact_columns(i["x"]))}
    if k == "route":
        return _exact_route(case, i)
    order, place, counts = _exact_plan(i["chosen"], case["E"])
    if k == "experts":
        x, N, K = _exact_rows(i["x"]), case["N"], case["K"]
        dev, train = x.device, case["train"]
        out = {"y": torch.zeros(order.numel(), N, dtype=torch.float64, device=dev)}
        if train:
            dy = _exact_rows(i["dy"])
            out["dx"] = torch.zeros(order.numel(), K, dtype=torch.float64, device=dev)
            out["dw"] = torch.zeros(case["E"], N, K, dtype=torch.float64, device=dev)
        ends = torch.cumsum(counts, 0).tolist()
        for e in range(case["E"]):
            lo, hi = ends[e] - int(counts[e]), ends[e]
            if lo == hi:
                continue
            w, tokens = _exact_weight(i["w"][e]), order[lo:hi].long() // case["k"]
            out["y"][lo:hi] = torch.mm(x[tokens], w.t().contiguous())
            if train:
                out["dx"][lo:hi] = torch.mm(dy[lo:hi], w)
                out["dw"][e] = torch.mm(_exact_columns(i["dy"][lo:hi]).t().contiguous(), _exact_columns(i["x"][tokens]))
        return out if train else out["y"]
    T, D, w = case["T"], case["D"], i["weights"].double()
    total = torch.zeros(T, D, dtype=torch.float64, device=w.device)
    if case["train"]:
        d = i["dout"].double()
        dy, dw = torch.zeros(T * case["k"], D, dtype=torch.float64, device=w.device), torch.zeros_like(w)
    for j in range(case["k"]):
        at = place[:, j].long()
        rows = i["y"][at].double()
        total += w[:, j:j + 1] * rows
        if case["train"]:
            dy[at] = w[:, j:j + 1] * d
            dw[:, j] = (d * rows).sum(1)
    return {"out": total, "dy": dy, "dw": dw} if case["train"] else total
