"""The operators of a quantized transformer block's linear and activation layers, as they are measured.

Four kinds of cases, each one pass of what a training or serving program does:

quant   a matrix to microscaled 4-bit floating point and back: blocks of 32 elements along a row (or, with "columns", down a
        column), a power-of-two scale per block, elements of one sign, two exponent and one mantissa bits; to the nearest
        value, or stochastically (gradients) from counter-based random numbers of a given seed.
linear  Y = X W^T with both operands in that format: W laid out once, X quantized in the call.  "stochastic": the data
        gradient dX = dY W of the same layer (X is then the output gradient, W the weights by columns).
ckpt    an activation saved in 8 bits (blocks of 32, power-of-two scales) and restored for the backward pass.
act     a gated or plain activation layer whose input is kept in 8 bits only: its forward pass, and its backward pass
        from what was kept.
wgrad   the weight gradient dY^T X of a linear layer whose input was kept in 8 bits.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # a small ragged matrix, where the launches count: a head's weights, a short batch
        {"name": "quant_rows_small", "kind": "quant", "rows": 77, "cols": 1000, "dtype": "fp32", "columns": False, "stochastic": False},
        # the output gradient of a wide layer, by columns and stochastically: as the filter side of a 4-bit product wants it
        {"name": "quant_columns_large", "kind": "quant", "rows": 16384, "cols": 4096, "dtype": "bf16", "columns": True, "stochastic": True},
        # serving: one token through an expanding layer
        {"name": "linear_one_token", "kind": "linear", "M": 1, "N": 8192, "K": 2048, "dtype": "bf16", "out": "bf16", "stochastic": False},
        # serving: a few requests at once through a contracting layer, results in fp32
        {"name": "linear_few_tokens", "kind": "linear", "M": 13, "N": 2048, "K": 8192, "dtype": "fp32", "out": "fp32", "stochastic": False},
        # training on a ragged number of tokens: the data gradient, stochastically rounded
        {"name": "linear_data_gradient", "kind": "linear", "M": 1777, "N": 2080, "K": 4096, "dtype": "bf16", "out": "fp32", "stochastic": True},
        # training: the largest product
        {"name": "linear_large", "kind": "linear", "M": 16384, "N": 8192, "K": 8192, "dtype": "bf16", "out": "bf16", "stochastic": False},
        # a short, odd activation kept for the backward pass
        {"name": "ckpt_small", "kind": "ckpt", "rows": 333, "cols": 1111, "dtype": "fp32"},
        # the input of a wide layer
        {"name": "ckpt_large", "kind": "ckpt", "rows": 32768, "cols": 8192, "dtype": "bf16"},
        # a plain activation of a small block
        {"name": "act_gelu_small", "kind": "act", "rows": 300, "cols": 2050, "dtype": "fp32", "act": "gelu", "gated": False},
        # the gated activation of a large block
        {"name": "act_swiglu_large", "kind": "act", "rows": 16384, "cols": 8192, "dtype": "bf16", "act": "silu", "gated": True},
        # a small layer whose gradient arrives in fp32, odd in every size
        {"name": "wgrad_small", "kind": "wgrad", "M": 1531, "N": 607, "K": 1100, "dtype": "fp32"},
        # the weight gradient of a wide layer
        {"name": "wgrad_large", "kind": "wgrad", "M": 16384, "N": 8192, "K": 4096, "dtype": "bf16"},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and n >= 64:
            n = n // 32 * 32
        return min(hi, n + 1 if n == 3072 else n)

    kind = rng.choice(["quant", "linear", "linear", "ckpt", "act", "wgrad"])
    dtype = rng.choice(["bf16", "fp32"])
    if kind == "quant":
        return {"kind": kind, "rows": size(1, 16384), "cols": size(32, 4096), "dtype": dtype, "columns": rng.random() < 0.5,
                "stochastic": rng.random() < 0.5}
    if kind == "linear":
        return {"kind": kind, "M": size(1, 16384), "N": size(64, 8192), "K": size(64, 8192), "dtype": dtype, "out": rng.choice(["bf16", "fp32"]),
                "stochastic": rng.random() < 0.3}
    if kind == "ckpt":
        return {"kind": kind, "rows": size(1, 16384), "cols": size(32, 8192), "dtype": dtype}
    if kind == "act":
        return {"kind": kind, "rows": size(1, 8192), "cols": size(32, 8192), "dtype": dtype, "act": rng.choice(["silu", "gelu"]), "gated": rng.random() < 0.5}
    return {"kind": kind, "M": size(1, 16384), "N": size(32, 4096), "K": size(32, 4096), "dtype": dtype}


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
    spread = 10 ** (-3 * torch.rand(cols, generator=g, device="cuda") - 1)
    return (-torch.sign(u) * torch.log1p(-2 * u.abs()).clamp_min(-16) * spread).to(DT[dtype])


def _weight(g, N, K):
    return (torch.randn(N, K, generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)


def _inputs(case, seed):
    g = _generator(seed)
    k = case["kind"]
    if k == "quant":
        make = _gradient if case["stochastic"] else _activation
        return {"x": make(g, case["rows"], case["cols"], case["dtype"])}
    if k == "linear":
        make = _gradient if case["stochastic"] else _activation
        return {"x": make(g, case["M"], case["K"], case["dtype"]), "w": _weight(g, case["N"], case["K"])}
    if k == "ckpt":
        return {"x": _activation(g, case["rows"], case["cols"], case["dtype"])}
    if k == "act":
        wide = case["cols"] * (2 if case["gated"] else 1)
        return {"h": _activation(g, case["rows"], wide, case["dtype"]), "dy": _gradient(g, case["rows"], case["cols"], case["dtype"])}
    return {"x": _activation(g, case["M"], case["K"], "bf16"), "dy": _gradient(g, case["M"], case["N"], case["dtype"])}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case, seed=seed)
    if own:
        from paper_2102_04782_amd import binding as daq

        s["daq"] = daq
        s["mode"] = daq.ROUND_STOCHASTIC if case.get("stochastic") else daq.ROUND_NEAREST
        if case["kind"] == "act":
            s["act"] = {"silu": daq.ACT_SILU, "gelu": daq.ACT_GELU}[case["act"]]
        if case["kind"] == "linear":     # laid out once, as a program keeps its weights
            s["w"] = daq.mx4_quantize(s["w"])
        if case["kind"] == "wgrad":      # what the forward pass has kept
            s["x"] = daq.ckpt8_save(s["x"])
    else:
        if case["kind"] == "linear":
            s["w"] = _mx4(s["w"], False, 0)
        if case["kind"] == "wgrad":
            s["x"] = _ckpt8(s["x"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _blocks(x):
    """[rows, cols] in 32 bits, as [rows, blocks, 32] with zeros behind the last column."""
    x = x.float()
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).reshape(x.shape[0], -1, 32)


def _power(e):
    """2^e of whole numbers -126 .. 127, in 32 bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(v):
    """floor(log2 v) of non-negative 32-bit values; -127 for zero and what is below the normal range."""
    return (v.view(torch.int32) >> 23).long() - 127


def _mix(h):
    """The 32-bit finalizer of MurmurHash3, on 64-bit integers that hold 32-bit values."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _draws(rows, cols, seed, device):
    """16 random bits for every element: neighbours in a row share a mixed word, the even column takes its upper half."""
    key = _mix(torch.tensor((seed & 0xFFFFFFFF) ^ int(_mix(torch.tensor((seed >> 32) ^ 0x9E3779B9)))))
    half = (cols + 1) // 2
    h = _mix(torch.arange(rows * half, device=device).view(rows, half) ^ int(key))
    return torch.stack((h >> 16, h & 0xFFFF), 2).view(rows, 2 * half)[:, :cols]


def _mx4(x, stochastic, seed, columns=False):
    """The values that x stands for in microscaled 4 bits, fp32."""
    rows, cols = x.shape
    u = _draws(rows, cols, seed, x.device).float() if stochastic else None
    if columns:
        x, u = x.t(), u.t() if stochastic else None
    b = _blocks(x)
    top = b.abs().amax(2, keepdim=True)
    e = _exponent(top) - 2
    if stochastic:                       # nothing is cut off: the largest value is at most 6 units
        e = e + ((top.view(torch.int32) & 0x7FFFFF) > 0x400000).long()
    e = e.clamp_min(-126)
    t = b.abs() * _power(-e)
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    if stochastic:
        n = torch.floor(t / step)
        v = (n + (torch.floor((t / step - n) * 65536) > _blocks(u)).float()) * step
    else:
        v = (torch.round(t / step) * step).clamp_max(6)
    v = torch.where(b < 0, -v, v) * _power(e)
    return v.view(v.shape[0], -1)[:, :x.shape[1]]


def _ckpt8(x):
    """8-bit codes and the exponents of their blocks."""
    b = _blocks(x)
    e = (_exponent(b.abs().amax(2, keepdim=True)) - 6).clamp_min(-126)
    return torch.round(b * _power(-e)).clamp(-127, 127).to(torch.int8), e, x.shape[1]


def _ckpt8_values(kept):
    codes, e, cols = kept
    v = codes.float() * _power(e)
    return v.view(v.shape[0], -1)[:, :cols]


def _act(x, name):
    """The activation function and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-x))
        return x * s, s * (1 + x * (1 - s))
    p = 0.5 * (1 + torch.erf(x * 0.5 ** 0.5))
    return x * p, p + x * torch.exp(-0.5 * x * x) * (0.5 / math.pi) ** 0.5


def _run_plain(s):
    case, k = s["case"], s["case"]["kind"]
    if k == "quant":
        return _mx4(s["x"], case["stochastic"], s["seed"], case["columns"]).to(s["x"].dtype)
    if k == "linear":
        return torch.matmul(_mx4(s["x"], case["stochastic"], s["seed"]), s["w"].t()).to(DT[case["out"]])
    if k == "ckpt":
        return _ckpt8_values(_ckpt8(s["x"])).to(s["x"].dtype)
    if k == "wgrad":
        return torch.matmul(s["dy"].float().t(), _ckpt8_values(s["x"]))
    h, dy, to = s["h"], s["dy"].float(), s["h"].dtype
    if not case["gated"]:
        y, _ = _act(h.float(), case["act"])
        _, slope = _act(_ckpt8_values(_ckpt8(h)), case["act"])
        return {"y": y.to(to), "dh": (dy * slope).to(to)}
    F = case["cols"]
    y = _act(h[:, :F].float(), case["act"])[0] * h[:, F:].float()
    gate, up = _ckpt8_values(_ckpt8(h[:, :F])), _ckpt8_values(_ckpt8(h[:, F:]))
    a, slope = _act(gate, case["act"])
    return {"y": y.to(to), "dh": torch.cat((dy * up * slope, dy * a), 1).to(to)}


def run(s):
    if not own:
        return _run_plain(s)
    daq, case, k = s["daq"], s["case"], s["case"]["kind"]
    if k == "quant":
        return daq.mx4_dequantize(daq.mx4_quantize(s["x"], transpose=case["columns"], mode=s["mode"], seed=s["seed"]), dtype=s["x"].dtype)
    if k == "linear":
        return daq.mx4_linear(s["x"], s["w"], mode=s["mode"], seed=s["seed"], dtype=DT[case["out"]])
    if k == "ckpt":
        return daq.ckpt8_restore(daq.ckpt8_save(s["x"]), dtype=s["x"].dtype)
    if k == "wgrad":
        return daq.ckpt8_weight_grad(s["dy"], s["x"])
    y, kept = daq.ckpt8_act_forward(s["h"], s["act"], gated=case["gated"])
    return {"y": y, "dh": daq.ckpt8_act_backward(s["dy"], kept, s["act"])}


def work(case):
    k = case["kind"]
    size = 2 if case["dtype"] == "bf16" else 4
    if k in ("quant", "ckpt"):
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * size * n, "flops": 4 * n}
    if k == "act":                       # input and output gradient, output and input gradient
        n, wide = case["rows"] * case["cols"], 2 if case["gated"] else 1
        return {"bytes": size * n * (2 + 2 * wide), "flops": 30 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if k == "linear":                    # 17 bytes for a block of 32 weights
        return {"bytes": size * M * K + N * -(-K // 32) * 17 + (2 if case["out"] == "bf16" else 4) * M * N, "flops": 2 * M * N * K}
    return {"bytes": size * M * N + M * -(-K // 32) * 33 + 4 * N * K, "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_scale(x, below):
    """x in blocks of 32, and 2^e per block, e = floor(log2 of the block's largest value) - below, both fp64."""
    x = x.double()
    rows, cols = x.shape
    full = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    full = full.reshape(rows, -1, 32)
    largest = full.abs().max(dim=2, keepdim=True).values
    e = torch.where(largest > 0, torch.frexp(largest)[1].double() - 1 - below, torch.full_like(largest, -126.0))
    return full, largest, e


def _exact_mx4(x, stochastic, seed, columns=False):
    rows, cols = x.shape
    u = None
    if stochastic:
        import numpy as np

        def mix(v):
            v = v.astype(np.uint32)
            v = (v ^ (v >> np.uint32(16))) * np.uint32(0x85EBCA6B)
            v = (v ^ (v >> np.uint32(13))) * np.uint32(0xC2B2AE35)
            return v ^ (v >> np.uint32(16))

        key = mix(np.array([seed & 0xFFFFFFFF], np.uint32) ^ mix(np.array([(seed >> 32) ^ 0x9E3779B9], np.uint32)))
        words = mix(np.arange(rows * ((cols + 1) // 2), dtype=np.uint32) ^ key).reshape(rows, -1)
        bits = np.empty((rows, 2 * words.shape[1]), np.float64)
        bits[:, 0::2], bits[:, 1::2] = words >> np.uint32(16), words & np.uint32(0xFFFF)
        u = torch.from_numpy(bits[:, :cols]).to(x.device)
    if columns:
        x, u = x.t(), None if u is None else u.t()
    full, largest, e = _exact_scale(x, 2)
    if stochastic:
        e = torch.where(largest > 6 * torch.exp2(e), e + 1, e)
    scale = torch.exp2(e.clamp(min=-126))
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    t = full.abs() / scale
    if stochastic:
        low = torch.bucketize(t, grid, right=True) - 1
        high = (low + 1).clamp(max=7)
        width = torch.where(high > low, grid[high] - grid[low], torch.ones_like(t))
        share = torch.floor((t - grid[low]) / width * 65536)
        draws = _exact_scale(u, 0)[0]
        index = torch.where(share > draws, high, low)
    else:
        middle = (grid[1:] + grid[:-1]) / 2
        index = torch.bucketize(t, middle)                  # a tie goes down ..
        tie = (index < 7) & (t == middle[index.clamp(max=6)]) & (index % 2 == 1)
        index = index + tie.long()                          # .. unless the upper one is the even code
    v = (torch.sign(full) * grid[index] * scale).reshape(full.shape[0], -1)
    return v[:, :x.shape[1]]


def _exact_ckpt8(x):
    full, _, e = _exact_scale(x, 6)
    scale = torch.exp2(e.clamp(min=-126))
    v = (torch.clamp(torch.round(full / scale), -127, 127) * scale).reshape(full.shape[0], -1)
    return v[:, :x.shape[1]]


def _exact_act(x, name, derivative):
    if name == "silu":
        s = torch.sigmoid(x)
        return s + x * s * torch.sigmoid(-x) if derivative else x * s
    phi = 0.5 * torch.special.erfc(-x / math.sqrt(2))
    return phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi) if derivative else x * phi


def exact(case, seed):
    i, k = _inputs(case, seed), case["kind"]
    if k == "quant":
        return _exact_mx4(i["x"], case["stochastic"], seed, case["columns"])
    if k == "linear":
        return _exact_mx4(i["x"], case["stochastic"], seed) @ _exact_mx4(i["w"], False, 0).t().contiguous()
    if k == "ckpt":
        return _exact_ckpt8(i["x"])
    if k == "wgrad":
        return i["dy"].double().t().contiguous() @ _exact_ckpt8(i["x"])
    h, dy, F = i["h"], i["dy"].double(), case["cols"]
    if not case["gated"]:
        return {"y": _exact_act(h.double(), case["act"], False), "dh": dy * _exact_act(_exact_ckpt8(h), case["act"], True)}
    y = _exact_act(h[:, :F].double(), case["act"], False) * h[:, F:].double()
    gate, up = _exact_ckpt8(h[:, :F]), _exact_ckpt8(h[:, F:])
    dh = torch.cat((dy * up * _exact_act(gate, case["act"], True), dy * _exact_act(gate, case["act"], False)), dim=1)
    return {"y": y, "dh": dh}
