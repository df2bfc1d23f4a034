"""Cases for timing the operators around a key-value cache held in 4 bits, each beside its plain form.

Three operators:
  tables   block tables and slot maps from the requests' lengths: pages are taken in order from a list of free ones, and
           every new token gets its request, its position and its slot in the cache
  append   rotary positions (one axis, or several as for images and video) on queries and keys, and the keys and values
           quantized into the pages of their slots; the values that the cache then holds come back beside the queries
  attend   attention of new tokens, one or many a request, over the pages of their requests, with the values that the
           cache's codes stand for

Definitions (decisions are taken on exact values, ties go to the even code):
  cache    blocks of 16 channels of a head: scale s = E4M3(max|block| / (6 t)), at most 448, element = nearest of 0, .5, 1,
           1.5, 2, 3, 4, 6 to x / (s t); t = 2^ceil(log2(amax / 2688)) from a known largest magnitude of keys and of values
  rotary   pair j of a head turns by pos[axis_j] * freq_j: a' = a cos - b sin, b' = b cos + a sin
  attend   o = softmax(scale q K^T) V over the positions that a token may see: not behind its own, and of those the last
           `window` where there is a window; a token that sees none has o = 0

With `own` set, run() calls the library; otherwise the same is formed by elementary torch operations.
"""
import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases ---------------------------------------------------------------------------------------
def listed():
    def tables(name, requests, new, long, held, page):
        return {"name": name, "op": "tables", "requests": requests, "new": new, "long": long, "held": held, "page": page, "mix": 1}

    def append(name, tokens, heads, kv_heads, dim, rotary, adjacent, sections, dtype, page):
        return {"name": name, "op": "append", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary,
                "adjacent": adjacent, "sections": sections, "dtype": dtype, "page": page}

    def attend(name, requests, new, long, held, heads, kv_heads, dim, window, dtype, page):
        return {"name": name, "op": "attend", "requests": requests, "new": new, "long": long, "held": held, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "window": window, "dtype": dtype, "page": page, "mix": 1}

    return [
        # sixty-four sequences that generate, a token each: latency
        tables("tables_generate", 64, 1, 0, 8192, 16),
        # a step of a busy server: prompts in pieces beside sequences that generate
        tables("tables_mixed", 1024, 1, 48, 4096, 32),
        # one generated token of a LLaMA-7B layer: latency
        append("append_one_token", 1, 32, 32, 128, 128, False, "", "f16", 16),
        # a prompt with images, positions of three axes, through a LLaMA-2-70B layer: bytes
        append("append_images", 8192, 64, 8, 128, 128, False, "16,24,24", "bf16", 64),
        # odd heads in binary32, turned in part, neighbouring channels a pair
        append("append_odd", 333, 12, 3, 80, 48, True, "", "f32", 16),
        # one generated token of a LLaMA-7B layer at the end of its context: latency
        attend("attend_one_token", 1, 1, 0, 4096, 32, 32, 128, 0, "f16", 16),
        # sixty-four sequences that generate in a LLaMA-2-70B layer: the cache's bytes
        attend("attend_generate", 64, 1, 0, 16384, 64, 8, 128, 0, "bf16", 64),
        # drafted tokens to be looked over, five a sequence
        attend("attend_drafted", 16, 5, 0, 8192, 64, 8, 128, 0, "bf16", 32),
        # sequences of odd lengths, some empty, small heads and a window
        attend("attend_window", 50, 1, 0, 6001, 20, 4, 64, 1000, "f16", 16),
        # a prompt of a LLaMA-7B layer: arithmetic
        attend("attend_prompt", 1, 4096, 0, 0, 32, 32, 128, 0, "bf16", 64),
        # a piece of a long prompt in a LLaMA-2-70B layer: arithmetic
        attend("attend_long_prompt", 1, 1024, 0, 32768, 64, 8, 128, 0, "bf16", 64),
        # pieces of prompts beside sequences that generate
        attend("attend_mixed", 24, 1, 3, 4000, 28, 4, 128, 0, "bf16", 16),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "attend"])
    page = rng.choice([16, 16, 32, 64, 128])
    if op == "tables":
        return {"op": op, "requests": _log(rng, 1, 2048), "new": rng.choice([0, 1, 1, 4]), "long": rng.choice([0, 5, 20]),
                "held": _log(rng, 1, 16384), "page": page, "mix": rng.randrange(1 << 20)}
    dim = rng.choice([64, 128, 128, 128, 16 * rng.randint(1, 16)])
    kv_heads = _log(rng, 1, 32)
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8, 8, 16])
    if op == "append":
        tokens = _log(rng, 1, 8192)
        while tokens * (heads + kv_heads) * dim > 8192 * 72 * 128:
            tokens = tokens // 2 + 1
        rotary = rng.choice([dim, dim, dim // 2])
        a, b = rotary // 8, rotary // 8 + rotary // 16
        sections = rng.choice(["", "", "%d,%d,%d" % (a, b, rotary // 2 - a - b)])
        return {"op": op, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "adjacent": rng.random() < 0.3,
                "sections": sections, "dtype": rng.choice(["f32", "f16", "bf16", "bf16"]), "page": page}
    kind = rng.choice(["generate", "generate", "drafted", "prompt", "mixed"])
    held = _log(rng, 1, 32768)
    if kind == "prompt":
        requests, new, long = rng.randint(1, 3), _log(rng, 2, 2048), 0
    else:
        requests, new, long = _log(rng, 1, 128), 1 if kind != "drafted" else rng.randint(2, 8), 0 if kind != "mixed" else rng.randint(1, 2)
    case = {"op": op, "requests": requests, "new": new, "long": long, "held": held, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "window": rng.choice([0, 0, 0, _log(rng, 1, 8192)]), "dtype": rng.choice(["f16", "bf16"]), "page": page, "mix": rng.randrange(1 << 20)}
    # what the plain form unpacks and the scores that it holds
    while True:
        past, fresh = _requests(case)
        most = max(p + n for p, n in zip(past, fresh))
        if case["requests"] * most * kv_heads * dim <= 64 * 16384 * 8 * 128 // 2 and case["requests"] * max(fresh) * most * heads <= 1 << 30:
            return case
        if case["requests"] > 4:
            case["requests"] = case["requests"] // 2 + 1
        elif case["held"] > 1000:
            case["held"] //= 2
        else:
            case["new"] = case["new"] // 2 + 1
            case["long"] = 0


def _requests(case):
    """Tokens held and new tokens of each request, from the case alone.  The first `long` requests bring pieces of prompts,
    some of the others nothing; lengths lie between an eighth of `held` and `held`, the first one's at it."""
    rng = random.Random(case["mix"])
    past, new = [], []
    for k in range(case["requests"]):
        held = case["held"] if k == 0 else rng.randint(case["held"] // 8, case["held"])
        if k < case["long"]:
            n = rng.randint(200, 700)
        elif case["op"] == "tables" or case["window"]:
            n = case["new"] if rng.random() < 0.9 else 0
        else:
            n = case["new"]
        if rng.random() < 0.04 and k:
            held = 0
        past.append(held)
        new.append(n)
    if not sum(new):
        new[0] = 1
    return past, new


# ---- inputs --------------------------------------------------------------------------------------
def _activations(gen, rows, heads, dim, dtype, loud):
    """Normal activations; of a head's channels a few are `loud` times as large, as keys have them."""
    x = torch.randn(rows, heads, dim, generator=gen, device="cuda")
    if loud:
        few = torch.rand(heads, dim, generator=gen, device="cuda") < 0.02
        x = x * torch.where(few, loud, 1.0)
    return x.to(_DTYPES[dtype])


def _pages_of(lengths, page):
    return [-(-n // page) for n in lengths]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    page = case["page"]
    if case["op"] == "append":
        t, d = case["tokens"], case["dim"]
        # one projection's result: queries, keys and values of a token lie side by side
        qkv = _activations(gen, t, case["heads"] + 2 * case["kv_heads"], d, case["dtype"], 8.0)
        pages = -(-t // page) + 1
        got = {"q": qkv[:, :case["heads"]], "k": qkv[:, case["heads"]:case["heads"] + case["kv_heads"]],
               "v": qkv[:, case["heads"] + case["kv_heads"]:], "pages": pages,
               "slots": torch.randperm(pages * page, generator=gen, device="cuda")[:t].int()}
        axes = case["sections"].count(",") + 1
        first = int(torch.randint(0, 100000, (1,), generator=gen, device="cuda"))
        at = torch.arange(first, first + t, device="cuda")
        # text goes on by one on every axis; an image's patches share a time and have a row and a column
        rows = [at, at // 64, at % 64 + first][:axes] if axes > 1 else [at]
        got["positions"] = torch.stack(rows).int()
        half = case["rotary"] // 2
        got["freq"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        sections = [int(s) for s in case["sections"].split(",")] if case["sections"] else [half]
        got["axis"] = torch.repeat_interleave(torch.arange(axes), torch.tensor(sections)).cuda()
        got["amax"] = (got["k"].abs().amax().float().reshape(1) * 1.5, got["v"].abs().amax().float().reshape(1))
        return got
    past, new = _requests(case)
    lengths = [p + n for p, n in zip(past, new)]
    held = _pages_of(past if case["op"] == "tables" else lengths, page)
    width, n_pages = max(_pages_of(lengths, page)) + 1, sum(_pages_of(lengths, page)) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").int()
    columns = torch.arange(width, device="cuda")
    counts = torch.tensor(held, device="cuda")
    first = counts.cumsum(0) - counts
    inside = columns[None] < counts[:, None]
    table = torch.where(inside, order[(first[:, None] + columns[None]).clamp(max=n_pages - 1)], -1).int()
    got = {"table": table, "past": torch.tensor(past, device="cuda").int(), "new": torch.tensor(new, device="cuda").int(),
           "pages": n_pages}
    if case["op"] == "tables":
        got["free"] = order[sum(held):].contiguous()
        return got
    got["lengths"] = torch.tensor(lengths, device="cuda").int()
    got["offsets"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    got["q"] = _activations(gen, sum(new), case["heads"], case["dim"], case["dtype"], 0)
    total = sum(lengths)
    got["k"] = _activations(gen, total, case["kv_heads"], case["dim"], case["dtype"], 6.0)
    got["v"] = _activations(gen, total, case["kv_heads"], case["dim"], case["dtype"], 0)
    got["amax"] = (got["k"].abs().amax().float().reshape(1), got["v"].abs().amax().float().reshape(1))
    owner = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), got["lengths"].long())
    starts = got["lengths"].long().cumsum(0) - got["lengths"]
    at = torch.arange(total, device="cuda") - starts[owner]
    got["slots"] = (table[owner, at // page] * page + at % page).int()
    return got


# ---- plain form ----------------------------------------------------------------------------------
def _tensor_scale(amax):
    """2^ceil(log2(amax / 2688)) as a tensor of one element."""
    mantissa, exponent = torch.frexp(amax.double() / 2688.0)
    return torch.ldexp(torch.ones_like(mantissa), exponent - (mantissa == 0.5).int())


def _plain_quantize(x, amax):
    """Codes (level numbers 0..7 with the sign as bit 3) and E4M3 scale bytes of [..., dim] in blocks of 16; decisions in 64 bits."""
    t = _tensor_scale(amax)
    x = x.double().unflatten(-1, (-1, 16))
    u = x.abs().amax(dim=-1) / (6.0 * t)
    step = torch.ldexp(torch.ones_like(u), torch.frexp(u.clamp(min=2.0 ** -6))[1] - 4)
    s = (torch.round(u / step) * step).clamp(max=448.0)
    y = torch.where(s[..., None] > 0, x / (s * t)[..., None], 0.0)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for edge, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if closed else (a > edge)
    code += (y < 0).to(torch.uint8) * 8
    return code.flatten(-2), s.float().to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_values(code, scale, amax):
    table = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=code.device)
    s = scale.view(torch.float8_e4m3fn).float() * _tensor_scale(amax).float()
    return (table[code.int()].unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _plain_pack(code):
    pairs = code.unflatten(-1, (-1, 2))
    return pairs[..., 0] | (pairs[..., 1] << 4)


def _plain_unpack(packed):
    return torch.stack((packed & 15, packed >> 4), dim=-1).flatten(-2)


def _plain_rotate(x, angle, adjacent):
    """x [tokens, heads, dim] in 64 bits turned by angle [tokens, pairs]."""
    half = angle.shape[1]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    x = x.double()
    if adjacent:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    else:
        a, b = x[..., :half], x[..., half:2 * half]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), dim=-1).flatten(-2) if adjacent else torch.cat((a, b), dim=-1)
    return torch.cat((turned, x[..., 2 * half:]), dim=-1)


def _plain_append(s):
    case = s["case"]
    angle = s["positions"][s["axis"]].T.double() * s["freq"]
    q = _plain_rotate(s["q"], angle, case["adjacent"]).to(s["q"].dtype)
    k = _plain_rotate(s["k"], angle, case["adjacent"])
    page, slots = case["page"], s["slots"].long()
    values = []
    for x, amax, codes, scales in ((k, s["amax"][0], s["k_codes"], s["k_scales"]), (s["v"], s["amax"][1], s["v_codes"], s["v_scales"])):
        code, scale = _plain_quantize(x, amax)
        codes[slots // page, :, slots % page] = _plain_pack(code)
        scales[slots // page, :, slots % page] = scale
        values.append(_plain_values(code, scale, amax).to(_values_dtype(case)))
    return [q] + values


def _plain_attend(s):
    case, q = s["case"], s["q"]
    h, page, d = case["kv_heads"], case["page"], case["dim"]
    most_new, longest = max(s["counts"][1]), max(p + n for p, n in zip(*s["counts"]))
    n_pages = max(1, -(-longest // page))
    pages = s["table"][:, :n_pages].clamp(min=0).long()
    k, v = (_plain_values(_plain_unpack(c[pages]), f[pages], a).permute(0, 2, 1, 3, 4).reshape(len(pages), h, -1, d)
            for c, f, a in ((s["k_codes"], s["k_scales"], s["amax"][0]), (s["v_codes"], s["v_scales"], s["amax"][1])))
    new = torch.arange(most_new, device=q.device)
    counts = (s["offsets"][1:] - s["offsets"][:-1]).long()
    inside = new[None] < counts[:, None]
    rows = (s["offsets"][:-1, None] + new[None]).clamp(max=len(q) - 1).long()
    group = case["heads"] // h
    qp = q[rows].float().unflatten(2, (h, group)).permute(0, 2, 3, 1, 4).reshape(len(pages), h, group * most_new, d)
    scores = (qp @ k.transpose(-1, -2)).mul_(d ** -0.5).unflatten(2, (group, most_new))
    position = torch.arange(k.shape[2], device=q.device)
    last = (s["lengths"].long() - counts)[:, None] + new[None]
    seen = position[None, None] <= last[..., None]
    if case["window"]:
        seen &= position[None, None] > last[..., None] - case["window"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    p = scores.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (group, most_new)) / torch.where(total > 0, total, 1.0)
    out = torch.zeros_like(q)
    out[rows[inside]] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[inside].to(q.dtype)
    return out


def _plain_tables(s):
    case, past, new = s["case"], s["past"].long(), s["new"].long()
    page, table, total = case["page"], s["table"], s["rows"]
    lengths = past + new
    had = (past + page - 1) // page
    need = (lengths + page - 1) // page - had
    before = need.cumsum(0) - need
    column = torch.arange(table.shape[1], device=table.device)[None] - had[:, None]
    fresh = (column >= 0) & (column < need[:, None])
    free = s["free"][(before[:, None] + column).clamp(0, len(s["free"]) - 1)]
    torch.where(fresh, free, table, out=table)
    offsets = torch.cat((new.new_zeros(1), new.cumsum(0)))
    row = torch.arange(total, device=table.device)
    request = torch.searchsorted(offsets, row, right=True) - 1
    position = past[request] + row - offsets[request]
    slots = table[request, position // page] * page + position % page
    return [table, lengths.int(), offsets.int(), request.int(), position.int(), slots.int(), need.sum().int().reshape(1)]


# ---- one pass ------------------------------------------------------------------------------------
def _values_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2309_15531_b200 import binding as B
    if case["op"] == "tables":
        s["rows"] = sum(_requests(case)[1])
        if own:
            s["plan"] = B.PageTables(case["requests"], s["rows"])
        return s
    h, page, d = case["kv_heads"], case["page"], case["dim"]
    if own:
        s["cache"] = B.Kv4Cache(s["pages"], page, h, d, k_amax=s["amax"][0], v_amax=s["amax"][1])
        if case["op"] == "append":
            s["rotary"] = B.Rotary(s["freq"], s["axis"], adjacent=case["adjacent"])
            s["out"] = (torch.empty(case["tokens"], case["heads"], d, dtype=s["q"].dtype, device="cuda"),
                        torch.empty(case["tokens"], h, d, dtype=_values_dtype(case), device="cuda"),
                        torch.empty(case["tokens"], h, d, dtype=_values_dtype(case), device="cuda"))
        else:
            B.kv4_append(s["k"], s["v"], s["cache"], s["slots"])
            s["max_new"] = max(_requests(case)[1])
            s["out"] = torch.empty_like(s["q"])
            s["workspace"] = torch.empty(B.kv4_workspace_bytes(case["requests"], len(s["q"]), case["heads"], h, d), dtype=torch.uint8, device="cuda")
    else:
        for name in ("k", "v"):
            s[name + "_codes"] = torch.zeros(s["pages"], h, page, d // 2, dtype=torch.uint8, device="cuda")
            s[name + "_scales"] = torch.zeros(s["pages"], h, page, d // 16, dtype=torch.uint8, device="cuda")
        if case["op"] == "attend":
            s["counts"] = _requests(case)
            for name, amax in zip(("k", "v"), s["amax"]):
                x, slots = s[name], s["slots"].long()
                for at in range(0, len(x), 65536):
                    code, scale = _plain_quantize(x[at:at + 65536], amax)
                    some = slots[at:at + 65536]
                    s[name + "_codes"][some // page, :, some % page] = _plain_pack(code)
                    s[name + "_scales"][some // page, :, some % page] = scale
    if case["op"] == "attend":
        for name in ("k", "v", "slots"):
            del s[name]                                  # what a program keeps is the cache
    return s


def run(s):
    case = s["case"]
    if not own:
        return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend}[case["op"]](s)
    from paper_2309_15531_b200 import binding as B
    if case["op"] == "tables":
        p = B.page_tables(s["past"], s["new"], s["table"], s["free"], case["page"], s["plan"])
        return [s["table"], p.lengths, p.offsets, p.requests, p.positions, p.slots, p.cursor]
    if case["op"] == "append":
        q, k_values, v_values = s["out"]
        B.kv4_append(s["k"], s["v"], s["cache"], s["slots"], q=s["q"], rotary=s["rotary"], positions=s["positions"], q_out=q,
                     k_values=k_values, v_values=v_values)
        return [q, k_values, v_values]
    return B.kv4_attention(s["q"], s["cache"], s["table"], s["lengths"], s["offsets"], window=case["window"], max_new=s["max_new"],
                           out=s["out"], workspace=s["workspace"])


def _seen(case):
    """For each request the positions that are read, and all pairs of a token and a position that it sees."""
    read, pairs = 0, 0
    w = case["window"]
    for p, n in zip(*_requests(case)):
        if n:
            read += min(p + n, w + n - 1) if w else p + n
            pairs += sum(min(p + j + 1, w) if w else p + j + 1 for j in range(n))
    return read, pairs


def work(case):
    """Inputs read once and outputs written once; of the cache what some token sees."""
    if case["op"] == "tables":
        past, new = _requests(case)
        taken = sum(_pages_of([p + n for p, n in zip(past, new)], case["page"])) - sum(_pages_of(past, case["page"]))
        return {"bytes": 4 * (4 * len(past) + 3 * sum(new) + 2 * taken + 2), "flops": 4 * sum(new) + 6 * len(past)}
    d, size = case["dim"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["op"] == "append":
        q, kv, t = case["heads"] * d, 2 * case["kv_heads"] * d, case["tokens"]
        return {"bytes": int(t * (q * 2 * size + kv * (size + 9 / 16 + (4 if size == 4 else 2)) + 8)), "flops": t * (3 * q + 12 * kv)}
    read, pairs = _seen(case)
    rows = sum(_requests(case)[1]) * case["heads"]
    return {"bytes": int(read * case["kv_heads"] * 2 * d * 9 / 16 + 2 * rows * d * size), "flops": 4 * pairs * case["heads"] * d}


# ---- in 64 bits ----------------------------------------------------------------------------------
def _exact_values(x, amax):
    """Q(x) from the definition in binary64, rounding on the grid that each magnitude falls on."""
    t = 2.0 ** math.ceil(math.log2(float(amax) / 2688.0))
    z = x.double().reshape(*x.shape[:-1], -1, 16)
    u = torch.maximum(z.amax(-1), -z.amin(-1)) / (6.0 * t)
    step = torch.exp2(torch.floor(torch.log2(u.clamp(min=2.0 ** -6))) - 3.0)
    scale = torch.round(u / step).mul(step).clamp(max=448.0) * t
    r = (z / scale[..., None]).nan_to_num(0.0, 0.0, 0.0).abs()
    step = torch.where(r < 2.0, 0.5, torch.where(r < 4.0, 1.0, 2.0))
    q = torch.round(r / step).mul(step).clamp(max=6.0)
    return (q * torch.sign(z) * scale[..., None]).reshape(x.shape)


def _exact_turned(x, got, adjacent):
    """Every pair as a complex number times e^(i angle)."""
    half = len(got["freq"])
    angle = got["positions"].double()[got["axis"], :].T * got["freq"][None]
    spin = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.double().clone()
    first = torch.arange(half, device=x.device)
    a, b = (2 * first, 2 * first + 1) if adjacent else (first, first + half)
    z = torch.complex(y[..., a], y[..., b]) * spin
    y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    got = _inputs(case, seed)
    if case["op"] == "tables":
        return None
    if case["op"] == "append":
        q, k = (_exact_turned(got[n], got, case["adjacent"]) for n in ("q", "k"))
        return [q, _exact_values(k, got["amax"][0]), _exact_values(got["v"], got["amax"][1])]
    past, new = _requests(case)
    out, at, row = torch.zeros(got["q"].shape, dtype=torch.float64, device="cuda"), 0, 0
    group = case["heads"] // case["kv_heads"]
    for p, n in zip(past, new):
        k, v = (_exact_values(got[name][at:at + p + n], a) for name, a in zip(("k", "v"), got["amax"]))
        at += p + n
        if not n:
            continue
        place = torch.arange(p + n, device="cuda")
        for head in range(case["heads"]):
            for some in range(0, n, 1024):
                own_place = p + torch.arange(some, min(n, some + 1024), device="cuda")
                score = got["q"][row + some:row + some + len(own_place), head].double() @ k[:, head // group].T / math.sqrt(case["dim"])
                hidden = place[None] > own_place[:, None]
                if case["window"]:
                    hidden |= place[None] <= own_place[:, None] - case["window"]
                weight = torch.softmax(score.masked_fill(hidden, -math.inf), dim=1)
                out[row + some:row + some + len(own_place), head] = weight @ v[:, head // group]
        row += n
    return out
