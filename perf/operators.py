"""Cases for timing the microscaled 4-bit floating point operators, each beside its plain form.

Three operators:
  quantize  a matrix to E2M1 codes with one scale for every 32 (MXFP4) or 16 (NVFP4) elements of a row; the
            values the codes and scales stand for come back beside them
  linear    y = Q(x) Q(W)^T for 4-bit weights that are kept, and activations that are quantized in the call
  experts   the same product for rows sorted by expert, every expert with a weight of its own; a row names
            the token it is gathered from, and the numbers of rows are known on the device only

Definitions (all decisions are taken on exact values, ties go to the even code):
  MXFP4  scale 2^(floor(log2 max|block|) - 2), not below 2^-127, element = nearest of 0, .5, 1, 1.5, 2, 3, 4, 6
         to x / scale
  NVFP4  tensor scale t = 2^ceil(log2(amax / 2688)) from a known largest magnitude `amax`; block scale
         s = E4M3(max|block| / (6 t)), at most 448; element = nearest level to x / (s t), 0 where s is 0

With `own` set, run() calls the library; otherwise the same is formed by elementary torch operations in binary32.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BLOCK = {"mx": 32, "nv": 16}


# ---- cases ---------------------------------------------------------------------------------------
def listed():
    def quantize(name, rows, cols, dtype, fmt, gap=0):
        return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "format": fmt, "gap": gap}

    def linear(name, tokens, inp, out, dtype, fmt, gap=0):
        return {"name": name, "op": "linear", "tokens": tokens, "in": inp, "out": out, "dtype": dtype, "format": fmt,
                "gap": gap}

    def experts(name, tokens, top, n, idle, inp, out, dtype, fmt):
        return {"name": name, "op": "experts", "tokens": tokens, "top": top, "experts": n, "idle": idle, "in": inp,
                "out": out, "dtype": dtype, "format": fmt}

    return [
        # the weight of a LLaMA-7B gate or up projection, quantized once when a model is prepared
        quantize("quantize_weight_nv", 11008, 4096, "f16", "nv"),
        # a prompt's activations in front of an attention projection, columns of a wider buffer
        quantize("quantize_prompt_mx", 2048, 4096, "bf16", "mx", 8192),
        # an odd binary32 matrix: rows that are not aligned and a last block that is not full
        quantize("quantize_odd_nv", 333, 5003, "f32", "nv"),
        # one generated token through a LLaMA-7B attention projection: latency
        linear("linear_one_token_nv", 1, 4096, 4096, "f16", "nv"),
        # sixteen sequences that generate, through a LLaMA-2-70B gate projection: the weight's bytes
        linear("linear_sixteen_mx", 16, 8192, 28672, "bf16", "mx"),
        # a few tokens through a small odd layer, binary32 in and out
        linear("linear_odd_nv", 77, 1336, 1001, "f32", "nv"),
        # a prompt through a LLaMA-7B up projection
        linear("linear_prompt_nv", 2048, 4096, 11008, "bf16", "nv"),
        # a batch of prompts through a LLaMA-2-70B gate projection: arithmetic
        linear("linear_large_mx", 8192, 8192, 28672, "bf16", "mx"),
        # sixty-four sequences that generate, two of thirty-two experts each: the weights' bytes
        experts("experts_generate_mx", 64, 2, 32, 5, 4096, 2048, "bf16", "mx"),
        # a prompt over eight experts of which one gets nothing
        experts("experts_prompt_nv", 4096, 2, 8, 1, 4096, 11008, "bf16", "nv"),
        # a few tokens over odd experts
        experts("experts_odd_nv", 150, 3, 6, 2, 1360, 712, "f16", "nv"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "experts", "experts"])
    case = {"op": op, "dtype": rng.choice(["f32", "f16", "bf16", "bf16"]), "format": rng.choice(["mx", "nv"])}
    if op == "quantize":
        rows, cols = _log(rng, 1, 16384), _log(rng, 16, 16384)
        while rows * cols > 11008 * 8192:
            rows = rows // 2 + 1
        case.update(rows=rows, cols=cols, gap=rng.choice([0, 0, 8, 512, 33]))
        return case
    inp = _log(rng, 128, 12288)
    if rng.random() < 0.6:
        inp = (inp + 127) // 128 * 128
    out = _log(rng, 64, 28672)
    if rng.random() < 0.5:
        out = (out + 63) // 64 * 64
    if op == "linear":
        tokens = _log(rng, 1, 8192)
        while inp * out > 8192 * 28672 or tokens * inp * out > 8192 * 8192 * 28672 or tokens * out > 8192 * 28672:
            tokens, out = (tokens + 1) // 2, out // 2 + 1
        case.update(tokens=tokens, out=out, gap=rng.choice([0, 0, 0, 64, 5]))
    else:
        n = _log(rng, 2, 64)
        top = rng.randint(1, min(n, 4))
        idle = rng.randint(0, (n - top) // 2)
        tokens = _log(rng, 1, 8192)
        while n * inp * out > 8 * 4096 * 11008:
            out = out // 2 + 1
            inp = (inp // 2 + 127) // 128 * 128 if n * inp * out > 8 * 4096 * 11008 and inp > 512 else inp
        while tokens * top * (inp + out) > 2 * 4096 * (4096 + 11008):
            tokens = tokens // 2 + 1
        case.update(tokens=tokens, out=out, top=top, experts=n, idle=idle)
    case["in"] = inp
    return case


def _rows_of_experts(case):
    """Rows of each expert in falling order, from the case alone: some experts are liked better, `idle` get nothing.
    No expert has more rows than there are tokens."""
    n, total = case["experts"] - case["idle"], case["tokens"] * case["top"]
    weight = [1.0 / (1.0 + 0.5 * k) for k in range(n)]
    rows = [min(case["tokens"], int(total * w / sum(weight))) for w in weight]
    left, k = total - sum(rows), 0
    while left > 0:
        take = min(case["tokens"] - rows[k], left if k else (left + 1) // 2)
        rows[k] += take
        left, k = left - take, (k + 1) % n
    return rows + [0] * case["idle"]


# ---- plain form ----------------------------------------------------------------------------------
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _tensor_scale(amax):
    """2^ceil(log2(amax / 2688)) as a binary32 tensor of one element."""
    mantissa, exponent = torch.frexp(amax.float() / 2688.0)
    return torch.ldexp(torch.ones_like(mantissa), exponent - (mantissa == 0.5).int())


def _plain_quantize(x, fmt, amax):
    """(level numbers 0..7 with the sign as bit 3, uint8 [rows, blocks * B]; scales binary32 [rows, blocks])."""
    size = _BLOCK[fmt]
    x = x.float()
    if x.shape[1] % size:
        x = torch.nn.functional.pad(x, (0, size - x.shape[1] % size))
    x = x.reshape(x.shape[0], -1, size)
    top = x.abs().amax(dim=2)
    if fmt == "mx":
        exponent = (torch.frexp(top)[1] - 3).clamp(min=-127)
        scale = torch.ldexp(torch.ones_like(top), torch.where(top > 0, exponent, -127))
    else:
        t = _tensor_scale(amax)
        scale = ((top / t) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn).float() * t
    y = torch.where(scale[..., None] > 0, x / scale[..., None], 0.0)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for bound, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= bound) if closed else (a > bound)
    code += (y < 0).to(torch.uint8) * 8
    return code.reshape(x.shape[0], -1), scale


def _plain_values(code, scale):
    """The binary32 values of codes [rows, blocks * B] and scales [rows, blocks]."""
    table = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=code.device)
    v = table[code.int()].reshape(code.shape[0], scale.shape[1], -1)
    return (v * scale[..., None]).reshape(code.shape[0], -1)


def _plain_pack(code, scale, fmt, amax):
    """Two codes to a byte, scales as bytes: what a program keeps of a weight."""
    pairs = code.reshape(code.shape[0], -1, 2)
    packed = pairs[..., 0] | (pairs[..., 1] << 4)
    if fmt == "mx":
        return packed, (torch.frexp(scale)[1] + 126).to(torch.uint8)
    return packed, (scale / _tensor_scale(amax)).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_unpack(packed, scales, fmt, amax):
    code = torch.stack((packed & 15, packed >> 4), dim=-1).reshape(packed.shape[0], -1)
    if fmt == "mx":
        scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    else:
        scale = scales.view(torch.float8_e4m3fn).float() * _tensor_scale(amax)
    return _plain_values(code, scale)


def _plain_product(x, weight, fmt, x_amax, w_amax):
    code, scale = _plain_quantize(x, fmt, x_amax)
    return _plain_values(code, scale) @ _plain_unpack(weight[0], weight[1], fmt, w_amax).T


# ---- inputs --------------------------------------------------------------------------------------
def _weight(gen, rows, cols):
    """Normal weights with one entry in a thousand from a heavy tail, as the library's synthetic layers have."""
    w = torch.randn(rows, cols, generator=gen, device="cuda") * 0.02
    heavy = torch.rand(rows, cols, generator=gen, device="cuda") < 0.001
    return torch.where(heavy, w * 6.0, w).half()


def _activations(gen, rows, cols, dtype, gap):
    """Normal activations with one channel in two hundred fifty to a hundred times as large, in the first `cols`
    columns of a buffer that is `gap` wider."""
    x = torch.randn(rows, cols + gap, generator=gen, device="cuda")
    loud = torch.rand(cols + gap, generator=gen, device="cuda") < 0.005
    gain = 50.0 + 50.0 * torch.rand(cols + gap, generator=gen, device="cuda")
    return (x * torch.where(loud, gain, 1.0)).to(_DTYPES[dtype])[:, :cols]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "quantize":
        # weights are what is quantized in f16, activations in the other types
        if case["dtype"] == "f16":
            x = _weight(gen, case["rows"], case["cols"] + case["gap"])[:, :case["cols"]]
        else:
            x = _activations(gen, case["rows"], case["cols"], case["dtype"], case["gap"])
        return {"x": x, "x_amax": x.abs().amax().float().reshape(1)}
    got = {"x": _activations(gen, case["tokens"], case["in"], case["dtype"], case.get("gap", 0))}
    got["x_amax"] = got["x"].abs().amax().float().reshape(1)
    if case["op"] == "linear":
        got["w"] = [_weight(gen, case["out"], case["in"])]
    else:
        rows = _rows_of_experts(case)
        order = torch.randperm(len(rows), generator=torch.Generator().manual_seed(seed)).tolist()
        rows = [rows[k] for k in order]
        got["rows"] = rows
        tokens = case["tokens"]
        picks = [torch.randperm(tokens, generator=gen, device="cuda")[:r].sort().values for r in rows]
        got["row_index"] = torch.cat(picks).int()
        got["offsets"] = torch.tensor([0] + rows, device="cuda").cumsum(0).int()
        got["w"] = [_weight(gen, case["out"], case["in"]) for _ in rows]
    got["w_amax"] = torch.stack([w.abs().amax().float() for w in got["w"]]).amax().reshape(1)
    return got


def _in_strips(rows, cols):
    step = max(1, (1 << 25) // cols)
    return [slice(r, min(rows, r + step)) for r in range(0, rows, step)]


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    fmt = case["format"]
    if case["op"] == "quantize":
        if own:
            from paper_2309_15531_b200 import binding as B
            state["q"] = B.Fp4Tensor(case["rows"], case["cols"], B.MXFP4 if fmt == "mx" else B.NVFP4)
            state["values"] = torch.empty(case["rows"], case["cols"], dtype=_values_dtype(case), device="cuda")
        return state
    rows = len(state["row_index"]) if case["op"] == "experts" else case["tokens"]
    weights = state.pop("w")
    if own:
        from paper_2309_15531_b200 import binding as B
        code = B.MXFP4 if fmt == "mx" else B.NVFP4
        n = len(weights) if case["op"] == "experts" else 0
        q = B.Fp4Tensor(case["out"], case["in"], code, experts=n)
        for k, w in enumerate(weights):
            B.quantize_fp4(w, code, amax=state["w_amax"], q=q.expert(k) if n else q)
        state["w"] = q
        state["y"] = torch.empty(rows, case["out"], dtype=_DTYPES[case["dtype"]], device="cuda")
        state["workspace"] = torch.empty(B.workspace_bytes(B.WS_FP4, rows, case["in"], 4, n), dtype=torch.uint8, device="cuda")
        state["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        state["w"] = []
        for w in weights:
            parts = [_plain_pack(*_plain_quantize(w[s], fmt, state["w_amax"]), fmt, state["w_amax"])
                     for s in _in_strips(*w.shape)]
            state["w"].append((torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])))
    return state


def _values_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    case, fmt = state["case"], state["case"]["format"]
    if own:
        from paper_2309_15531_b200 import binding as B
        code = B.MXFP4 if fmt == "mx" else B.NVFP4
        if case["op"] == "quantize":
            B.quantize_fp4(state["x"], code, amax=state["x_amax"], q=state["q"], values=state["values"])
            return state["values"]
        if case["op"] == "linear":
            return B.fp4_linear(state["x"], state["w"], x_amax=state["x_amax"], y=state["y"],
                                workspace=state["workspace"], status=state["status"])
        return B.fp4_linear_grouped(state["x"], state["offsets"], state["w"], row_index=state["row_index"],
                                    x_amax=state["x_amax"], y=state["y"], workspace=state["workspace"],
                                    status=state["status"])
    x = state["x"]
    if case["op"] == "quantize":
        return _plain_values(*_plain_quantize(x, fmt, state["x_amax"]))[:, :x.shape[1]].to(_values_dtype(case))
    if case["op"] == "linear":
        return _plain_product(x, state["w"][0], fmt, state["x_amax"], state["w_amax"]).to(x.dtype)
    y = torch.empty(len(state["row_index"]), case["out"], dtype=x.dtype, device=x.device)
    at = 0
    for n, weight in zip(state["rows"], state["w"]):
        if n:
            rows = x[state["row_index"][at:at + n]]
            y[at:at + n] = _plain_product(rows, weight, fmt, state["x_amax"], state["w_amax"]).to(x.dtype)
        at += n
    return y


def work(case):
    """Inputs read once and outputs written once: 4-bit codes with their scales, and the experts that get rows."""
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    scaled = 0.5 + 1.0 / _BLOCK[case["format"]]
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": int(n * (size + scaled + (4 if case["dtype"] == "f32" else 2))), "flops": 4 * n}
    if case["op"] == "linear":
        weights, rows = 1, case["tokens"]
    else:
        counts = _rows_of_experts(case)
        weights, rows = sum(1 for n in counts if n), sum(counts)
    moved = weights * case["out"] * case["in"] * scaled + case["tokens"] * case["in"] * size + rows * case["out"] * size
    return {"bytes": int(moved), "flops": 2 * rows * case["in"] * case["out"]}


# ---- in 64 bits ----------------------------------------------------------------------------------
def _exact_values(x, fmt, amax):
    """Q(x) from the definition, in binary64 (rounding on the grid that each magnitude falls on)."""
    rows, cols = x.shape
    size = _BLOCK[fmt]
    blocks = -(-cols // size)
    z = torch.zeros(rows, blocks * size, dtype=torch.float64, device=x.device)
    z[:, :cols] = x.double()
    z = z.view(rows, blocks, size)
    top = torch.maximum(z.amax(2), -z.amin(2))
    if fmt == "mx":
        scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2.0)
        # the logarithm may round up to a whole number just below a power of two
        scale = torch.where(4.0 * scale > top, torch.where(scale > 2.0 ** -127, scale / 2.0, scale), scale)
        scale = torch.where(8.0 * scale <= top, scale * 2.0, scale)
    else:
        t = 2.0 ** math.ceil(math.log2(float(amax) / 2688.0))
        u = top / (6.0 * t)
        step = torch.exp2(torch.floor(torch.log2(u.clamp(min=2.0 ** -6))) - 3.0)
        scale = torch.round(u / step).mul(step).clamp(max=448.0) * t
    r = (z / scale[..., None]).nan_to_num(0.0, 0.0, 0.0).abs()
    step = torch.where(r < 2.0, 0.5, torch.where(r < 4.0, 1.0, 2.0))
    q = torch.round(r / step).mul(step).clamp(max=6.0)
    return (q * torch.sign(z) * scale[..., None]).view(rows, -1)[:, :cols]


def exact(case, seed):
    got = _inputs(case, seed)
    fmt, x = case["format"], got["x"]

    def values(m, amax):
        return torch.cat([_exact_values(m[s], fmt, amax) for s in _in_strips(*m.shape)])

    if case["op"] == "quantize":
        return values(x, got["x_amax"])
    xq = values(x, got["x_amax"])
    if case["op"] == "linear":
        return xq @ values(got["w"][0], got["w_amax"]).T
    parts, at = [], 0
    for n, w in zip(got["rows"], got["w"]):
        if n:
            parts.append(xq[got["row_index"][at:at + n].long()] @ values(w, got["w_amax"]).T)
        at += n
    return torch.cat(parts)
