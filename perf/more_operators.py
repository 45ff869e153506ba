"""Timed cases of the 4-bit token operators: append_tokens, attend_tokens, linear4.

Decoding with 4-bit state: keys and values are transformed (Sylvester blocks along
the head), quantized to 4 bits with one scale per token and head and written into
pages of a cache; attention reads that cache; projections multiply with 4-bit
weights that have one scale per group of inputs.

A page of the cache holds, per head, page x width / 2 bytes of key codes, as many of
value codes, then page float32 key scales and page float32 value scales. A byte holds
the codes + 8 of two neighbouring values, the first in its low half.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # one decoded token of each of 128 sequences goes into the cache: latency counts
        {"name": "append_decode_batch", "op": "append", "seqs": 128, "tokens": 1, "length": 4096, "kv": 8, "d": 128,
         "page": 64, "hb": 128, "dtype": "bf16"},
        # prompts of a few sequences, ragged, their values as the cache holds them handed back
        {"name": "append_prompts", "op": "append", "seqs": 4, "tokens": 4096, "length": 4096, "kv": 8, "d": 128,
         "page": 64, "hb": 128, "dtype": "bf16"},
        # single precision, small pages, three heads of a width that is no power of two
        {"name": "append_odd", "op": "append", "seqs": 5, "tokens": 333, "length": 777, "kv": 3, "d": 192,
         "page": 16, "hb": 64, "dtype": "f32"},
        # one token of a short conversation: latency counts
        {"name": "attend_one_token", "op": "attend", "seqs": 1, "tokens": 1, "length": 1000, "heads": 32, "kv": 8, "d": 128,
         "page": 64, "hb": 128, "dtype": "bf16"},
        # one token behind a long document
        {"name": "attend_long_document", "op": "attend", "seqs": 1, "tokens": 1, "length": 131072, "heads": 32, "kv": 8,
         "d": 128, "page": 64, "hb": 128, "dtype": "bf16"},
        # a decode batch of ragged sequences
        {"name": "attend_decode_batch", "op": "attend", "seqs": 64, "tokens": 1, "length": 8192, "heads": 32, "kv": 8,
         "d": 128, "page": 64, "hb": 128, "dtype": "bf16"},
        # a few drafted tokens each to be checked, every head its own keys, small pages
        {"name": "attend_drafts", "op": "attend", "seqs": 16, "tokens": 5, "length": 2050, "heads": 16, "kv": 16, "d": 64,
         "page": 16, "hb": 64, "dtype": "f16"},
        # a piece of a prompt behind earlier pieces of two sequences
        {"name": "attend_prompt_piece", "op": "attend", "seqs": 2, "tokens": 2048, "length": 8192, "heads": 32, "kv": 8,
         "d": 128, "page": 64, "hb": 128, "dtype": "bf16"},
        # one decoded token through a square projection: the weights' bytes and the latency count
        {"name": "linear4_one_token", "op": "linear4", "rows": 1, "k": 4096, "n": 4096, "group": 128, "x": "bf16",
         "out": "bf16", "codes": False, "bias": False},
        # a decode batch through an up projection
        {"name": "linear4_decode_batch", "op": "linear4", "rows": 16, "k": 4096, "n": 16384, "group": 128, "x": "bf16",
         "out": "bf16", "codes": False, "bias": False},
        # odd sizes all over, single precision, small groups, the last one cut
        {"name": "linear4_odd", "op": "linear4", "rows": 5, "k": 1000, "n": 1234, "group": 32, "x": "f32",
         "out": "f32", "codes": False, "bias": True},
        # a larger batch of tokens that were quantized to 8 bits, through a down projection
        {"name": "linear4_codes", "op": "linear4", "rows": 64, "k": 8192, "n": 4096, "group": 64, "x": "f16",
         "out": "bf16", "codes": True, "bias": False},
    ]


def _log(rng, lo, hi):
    """A size spread evenly over its logarithm: odd, a power of two, or a multiple of 160."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.randrange(3)
    v = v | 1 if kind == 0 else 1 << int(round(math.log2(v))) if kind == 1 else v // 160 * 160
    return min(hi, max(lo, v))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "linear4", "linear4"])
    if op == "linear4":
        k, n, codes = _log(rng, 64, 16384), _log(rng, 64, 16384), rng.random() < 0.3
        x = "f16" if codes else rng.choice(["bf16", "bf16", "f16", "f32"])
        return {"op": op, "rows": _log(rng, 1, 64), "k": k, "n": n, "group": rng.choice([32, 64, 128]), "x": x,
                "out": rng.choice(["bf16", "f16", "f32"]), "codes": codes, "bias": rng.random() < 0.5}
    d = rng.choice([64, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 16])
    case = {"op": op, "seqs": _log(rng, 1, 128), "tokens": 1, "length": 1, "kv": kv, "d": d,
            "page": rng.choice([16, 32, 64, 64]), "hb": rng.choice([1, 32, 64, d & -d]),
            "dtype": rng.choice(["bf16", "bf16", "f16"] + ["f32"] * (op == "append"))}
    # keys of all sequences together no more than the long document's
    most = max(1, min(131072, 131072 * 8 * 128 // (case["seqs"] * kv * d)))
    case["length"] = _log(rng, 1, most)
    if op == "append":
        if rng.random() < 0.5:
            case["tokens"] = min(case["length"], _log(rng, 1, max(1, 16384 * 8 * 128 // (case["seqs"] * kv * d))))
        return case
    case["heads"] = kv * rng.choice([1, 1, 2, 4, 4, 5, 7, 8, 16])
    kind = rng.random()
    if kind > 0.5:
        # a few tokens each, or pieces of prompts: products of queries and keys no more than the listed piece's
        room = 2 * 2048 * 8192 * 32 * 128 // (case["seqs"] * case["length"] * case["heads"] * d)
        case["tokens"] = max(1, min(case["length"], room, _log(rng, 2, 8) if kind < 0.75 else _log(rng, 8, 4096)))
    return case


# ------------------------------------------------------------------ ragged sequences

def _lengths(case):
    """Lengths of the sequences, new tokens included: spread from a sixteenth of the longest, which comes first."""
    part = [1 - 15 / 16 * (i * 0.618034 % 1) for i in range(case["seqs"])]
    return [max(1, round(case["length"] * p)) for p in part]


def _new(case):
    """New tokens of each sequence: 1, or spread up to the most of them."""
    part = [1 - 3 / 4 * (i * 0.754878 % 1) for i in range(case["seqs"])]
    return [max(1, min(n, round(case["tokens"] * p))) for n, p in zip(_lengths(case), part)]


def work(case):
    if case["op"] == "linear4":
        rows, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": n * ((k + 1) // 2 + 4 * -(-k // case["group"]) + 4 * case["bias"]) + rows * k * SIZE[case["x"]]
                + 4 * rows * case["codes"] + rows * n * SIZE[case["out"]], "flops": 2 * rows * n * k}
    lengths, new = _lengths(case), _new(case)
    kv, d, size = case["kv"], case["d"], SIZE[case["dtype"]]
    tables = 4 * sum(2 + -(-n // case["page"]) for n in lengths)
    if case["op"] == "append":
        values = 2 * sum(new) * kv * d                       # keys and values; in, the cache, and handed back
        return {"bytes": values * 2 * size + sum(new) * kv * (d + 8) + tables,
                "flops": values * (2 * math.log2(case["hb"]) + 5)}
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lengths, new))
    return {"bytes": sum(lengths) * kv * (d + 8) + 2 * sum(new) * case["heads"] * d * size + tables,
            "flops": 4 * pairs * case["heads"] * d}


# ------------------------------------------------------------------ inputs

def _hadamard(hb):
    h = torch.ones(1, 1, device="cuda")
    while h.shape[0] < hb:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h


def _codes4(g, *shape, low=-7):
    """Gaussian codes as a symmetric 4-bit quantizer leaves them."""
    return torch.randn(*shape, generator=g, device="cuda").mul_(2.6).round_().clamp_(low, 7).to(torch.int8)


def _cache(case, g, pages):
    """Pages of random codes and scales: keys of about unit size, values of different sizes from token to token."""
    kv, d, page = case["kv"], case["d"], case["page"]
    data = torch.empty(pages, kv, page * (d + 8), dtype=torch.uint8, device="cuda")
    for part in range(2):                                    # key codes, value codes
        c = (_codes4(g, pages, kv, page * d) + 8).to(torch.uint8)
        data[:, :, part * page * d // 2:(part + 1) * page * d // 2] = c[:, :, 0::2] | c[:, :, 1::2] << 4
    scales = 0.4 * torch.exp(0.3 * torch.randn(pages, kv, 2 * page, generator=g, device="cuda"))
    data[:, :, page * d:] = scales.view(torch.uint8)
    return data


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "linear4":
        rows, k, n = case["rows"], case["k"], case["n"]
        groups = -(-k // case["group"])
        s["sx"] = None
        if case["codes"]:                                    # 8-bit codes of a token quantizer and their scales
            s["x"] = (torch.randn(rows, k, generator=g, device="cuda") * 34).round_().clamp_(-127, 127).half()
            s["sx"] = 0.02 * torch.exp(0.3 * torch.randn(rows, generator=g, device="cuda"))
        else:
            # a channel's own spread, and a few outlier channels, as activations have them
            spread = torch.exp(0.5 * torch.randn(k, generator=g, device="cuda"))
            spread[torch.randint(0, k, (4,), generator=g, device="cuda")] *= 20
            s["x"] = (torch.randn(rows, k, generator=g, device="cuda") * spread).to(DTYPES[case["x"]])
        s["w"] = _codes4(g, n, k, low=-8)
        s["sw"] = 0.01 * torch.exp(0.3 * torch.randn(n, groups, generator=g, device="cuda"))
        s["b"] = torch.randn(n, generator=g, device="cuda") if case["bias"] else None
        if own:
            from paper_2608_01653_gb300 import hatq
            s["layer"] = hatq.prepare_linear4(s["w"], group=case["group"], scales=s["sw"], bias=s["b"])
        return s
    kv, d, page, dtype = case["kv"], case["d"], case["page"], DTYPES[case["dtype"]]
    lengths, new = torch.tensor(_lengths(case)), torch.tensor(_new(case))
    used = (lengths + page - 1) // page
    width, pages = int(used.max()), int(used.sum())
    # every sequence's pages lie anywhere in the cache; a few pages belong to nobody
    order = torch.randperm(pages + 3, generator=g, device="cuda").to(torch.int32)
    held = torch.arange(width)[None, :] < used[:, None]
    place = (torch.cumsum(held.flatten(), 0) - 1).reshape(held.shape).clamp(min=0)
    s["table"] = torch.where(held.cuda(), order[place.cuda()], -1)
    s["lengths"] = lengths.to(torch.int32).cuda()
    s["starts"] = None if case["tokens"] == 1 else torch.cat([new.new_zeros(1), torch.cumsum(new, 0)]).to(torch.int32).cuda()
    rows, s["most"] = int(new.sum()), int(new.max())
    s["data"] = _cache(case, g, pages + 3)
    s["h"] = _hadamard(case["hb"])
    if case["op"] == "append":
        spread = torch.exp(0.5 * torch.randn(2, kv, d, generator=g, device="cuda"))
        spread[:, :, torch.randint(0, d, (3,), generator=g, device="cuda")] *= 8
        s["k"], s["v"] = ((torch.randn(rows, kv, d, generator=g, device="cuda") * spread[i]).to(dtype) for i in range(2))
    else:
        s["q"] = torch.randn(rows, case["heads"], d, generator=g, device="cuda").to(dtype)
    if own:
        from paper_2608_01653_gb300 import hatq
        s["cache"] = hatq.TokenCache(s["data"], page=page, hb=case["hb"])
    return s


# ------------------------------------------------------------------ the operators

def _rows(s):
    """Sequence and position of every new token."""
    lengths = s["lengths"].long()
    if s["starts"] is None:
        return torch.arange(s["seqs"], device=lengths.device), lengths - 1
    starts = s["starts"].long()
    r = torch.arange((s["k"] if s["op"] == "append" else s["q"]).shape[0], device=lengths.device)
    b = torch.searchsorted(starts, r, right=True) - 1
    return b, lengths[b] - starts[b + 1] + r


def _quantize4(x, hb):
    """Sums and differences in fp32, shortest distances first; codes, scales and the values they stand for."""
    t, h = x.float(), 1
    while h < hb:
        a, b = t.reshape(*x.shape[:-1], -1, 2, h).unbind(-2)
        t, h = torch.stack([a + b, a - b], -2).reshape(x.shape), 2 * h
    most = t.abs().amax(-1, keepdim=True)
    codes = torch.where(most > 0, (7 * t / most).round(), 0)
    step = torch.where(most > 0, most / torch.full_like(most, 7), 1) * (1 / math.sqrt(hb))
    return codes, step


def _append(s):
    b, at = _rows(s)
    page, d, hb = s["page"], s["d"], s["hb"]
    block = s["table"][b, at // page].long()[:, None]
    head, slot = torch.arange(s["kv"], device=b.device)[None, :], (at % page)[:, None]
    codes, scales = s["data"][:, :, :page * d], s["data"][:, :, page * d:].view(torch.float32)

    def put(x, part):
        c, step = _quantize4(x, hb)
        n = (c + 8).to(torch.uint8)
        codes.unflatten(2, (2, page, d // 2))[block, head, part, slot] = n[:, :, 0::2] | n[:, :, 1::2] << 4
        scales.unflatten(2, (2, page))[block, head, part, slot] = step[:, :, 0]
        t = (c.reshape(-1, hb) @ s["h"]).reshape(c.shape) if hb > 1 else c
        return (t * (step * (1 / math.sqrt(hb)))).to(x.dtype)

    return put(s["k"], 0), put(s["v"], 1)


def _attend(s):
    page, d, kv, hb = s["page"], s["d"], s["kv"], s["hb"]
    seqs, width = s["table"].shape
    group = s["heads"] // kv
    got = s["data"][s["table"].clamp(min=0).long()].transpose(1, 2)            # [seqs][kv][width][...]
    scales = got[..., page * d:].contiguous().view(torch.float32)
    n = got[..., :page * d].reshape(seqs, kv, width, 2, page, d // 2)
    c = torch.stack([n & 15, n >> 4], -1).float().flatten(-2) - 8
    c *= scales.reshape(seqs, kv, width, 2, page, 1)
    k, v = (c[:, :, :, i].reshape(seqs, kv, width * page, d) for i in range(2))
    b, at = _rows(s)
    i = at - s["lengths"][b] + s["most"]                                       # the newest token of each comes last
    q = (s["q"].float().reshape(-1, hb) @ s["h"] / math.sqrt(hb)).reshape(-1, kv, group, d)
    padded = q.new_zeros(seqs, s["most"], kv, group, d)
    padded[b, i] = q
    w = padded.permute(0, 2, 1, 3, 4).reshape(seqs, kv, -1, d) @ k.transpose(2, 3)
    w = w.reshape(seqs, kv, s["most"], group, -1) * d ** -0.5
    last = s["lengths"][:, None] - s["most"] + torch.arange(s["most"], device=b.device)
    seen = torch.arange(width * page, device=b.device) <= last[:, :, None]
    w = w.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    o = w.reshape(seqs, kv, -1, width * page) @ v / w.sum(-1).reshape(seqs, kv, -1, 1)
    o = o.reshape(seqs, kv, s["most"], group, d).permute(0, 2, 1, 3, 4)[b, i]
    return (o.reshape(-1, hb) @ s["h"] / math.sqrt(hb)).reshape(s["q"].shape).to(s["q"].dtype)


def _linear4(s):
    w = s["w"].float() * torch.repeat_interleave(s["sw"], s["group"], 1)[:, :s["k"]]
    y = s["x"].float() @ w.T
    if s["sx"] is not None:
        y = y * s["sx"][:, None]
    return (y if s["b"] is None else y + s["b"]).to(DTYPES[s["out"]])


def run(s):
    op = s["op"]
    if not own:
        return {"append": _append, "attend": _attend, "linear4": _linear4}[op](s)
    from paper_2608_01653_gb300 import hatq
    if op == "append":
        return hatq.append_tokens(s["cache"], s["k"], s["v"], s["table"], s["lengths"], s["starts"], kept=True)
    if op == "attend":
        return hatq.attend_tokens(s["q"], s["cache"], s["table"], s["lengths"], s["starts"])
    return hatq.linear4(s["x"], s["layer"], scales=s["sx"], dtype=DTYPES[s["out"]])


# ------------------------------------------------------------------ the definitions in 64 bits

def _basis(hb):
    """The orthonormal Sylvester matrix by the parity of i & j."""
    i = torch.arange(hb)
    both = i[:, None] & i[None, :]
    parity = sum((both >> j) & 1 for j in range(9)) % 2
    return ((1.0 - 2.0 * parity) / math.sqrt(hb)).double().cuda()


def _turn(x, hb):
    return torch.einsum("...ij,jk->...ik", x.reshape(*x.shape[:-1], -1, hb), _basis(hb)).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    hb = case["hb"] if "hb" in case else 1
    if case["op"] == "linear4":
        y = torch.empty(case["rows"], case["n"], dtype=torch.float64, device="cuda")
        group = torch.arange(case["k"], device="cuda") // case["group"]
        for i in range(0, case["n"], 1024):
            y[:, i:i + 1024] = s["x"].double() @ (s["w"][i:i + 1024].double() * s["sw"][i:i + 1024].double()[:, group]).T
        if case["codes"]:
            y *= s["sx"].double()[:, None]
        return y + s["b"].double() if case["bias"] else y
    if case["op"] == "append":
        kept = []
        for x in (s["k"], s["v"]):
            t = _turn(x.double(), hb)
            step = t.abs().amax(-1, keepdim=True) / 7
            step[step == 0] = 1
            kept.append(_turn(torch.round(t / step) * step, hb))
        return tuple(kept)
    page, d, kv, group = case["page"], case["d"], case["kv"], case["heads"] // case["kv"]
    q, out, first = s["q"].double(), [], 0
    for b, (length, m) in enumerate(zip(_lengths(case), _new(case))):
        pages = s["data"][s["table"][b, :-(-length // page)].long()]
        scales = pages[:, :, page * d:].contiguous().view(torch.float32).double()
        for h in range(kv):
            held = []
            for part in range(2):
                n = pages[:, h, part * page * d // 2:(part + 1) * page * d // 2].reshape(-1, d // 2, 1)
                c = torch.cat([n % 16, n // 16], 2).reshape(-1, d).double() - 8
                held.append(_turn(c * scales[:, h, part * page:(part + 1) * page].reshape(-1, 1), hb)[:length])
            for i in range(0, m, 512):
                j = min(m, i + 512)
                x = q[first + i:first + j, h * group:(h + 1) * group]
                w = torch.einsum("mgd,nd->mgn", x, held[0]) / math.sqrt(d)
                late = torch.arange(length, device="cuda") > torch.arange(i, j, device="cuda")[:, None] + length - m
                w = torch.softmax(w.masked_fill(late[:, None, :], -math.inf), -1)
                out.append((first + i, h, torch.einsum("mgn,nd->mgd", w, held[1])))
        first += m
    y = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for r, h, o in out:
        y[r:r + o.shape[0], h * group:(h + 1) * group] = o
    return y
