"""Timed cases of the token operators: quantize_tokens, linear, grouped_linear, combine_rows.

A token layer in 8-bit integers: activations are transformed and quantized with
one scale per token, multiplied exactly with INT8 weights that have one scale
per output channel, either by one weight matrix or by the matrix of the expert
that a row was sent to, and expert rows are added up again per token.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1}


def listed():
    return [
        # the down projection's operand of one decoded token: gate and up halves in, codes out
        {"name": "quantize_one_token_gated", "op": "quantize", "rows": 1, "src": 1, "c": 8192, "hb": 256,
         "dtype": "bf16", "act": "silu", "gated": True, "gather": False, "codes": "f16"},
        # the operand of a prompt's projections
        {"name": "quantize_prompt", "op": "quantize", "rows": 8192, "src": 8192, "c": 4096, "hb": 128,
         "dtype": "bf16", "act": "none", "gated": False, "gather": False, "codes": "f16"},
        # a prompt's tokens copied to four experts each, some slots of the expert buffer empty, width with a ragged end
        {"name": "quantize_expert_rows", "op": "quantize", "rows": 16384, "src": 4096, "c": 2000, "hb": 16,
         "dtype": "f32", "act": "none", "gated": False, "gather": True, "codes": "f16"},
        # one decoded token through a square projection: the weights' bytes and the latency count
        {"name": "linear_one_token", "op": "linear", "rows": 1, "k": 4096, "n": 4096, "codes": "i8",
         "out": "bf16", "bias": False},
        # a decode batch through an up projection
        {"name": "linear_decode_batch", "op": "linear", "rows": 48, "k": 4096, "n": 8192, "codes": "f16",
         "out": "bf16", "bias": False},
        # odd sizes all over, single precision out, codes held in 8 bits
        {"name": "linear_odd", "op": "linear", "rows": 777, "k": 1000, "n": 1234, "codes": "i8",
         "out": "f32", "bias": True},
        # a prompt through an up projection
        {"name": "linear_prompt", "op": "linear", "rows": 8192, "k": 4096, "n": 16384, "codes": "f16",
         "out": "bf16", "bias": False},
        # one decoded token at its eight experts
        {"name": "experts_one_token", "op": "grouped", "rows": 8, "experts": 64, "active": 8, "k": 2048, "n": 1536,
         "codes": "i8", "out": "bf16", "bias": False},
        # 32 decoded tokens at eight experts each
        {"name": "experts_decode_batch", "op": "grouped", "rows": 256, "experts": 64, "active": 61, "k": 2048,
         "n": 2048, "codes": "f16", "out": "bf16", "bias": False},
        # a prompt at eight experts each, ragged, two experts idle
        {"name": "experts_prompt", "op": "grouped", "rows": 32768, "experts": 64, "active": 62, "k": 2048, "n": 1536,
         "codes": "f16", "out": "f16", "bias": False},
        # the way back to tokens: a decode batch and a prompt
        {"name": "combine_decode_batch", "op": "combine", "tokens": 32, "topk": 8, "c": 2048, "dtype": "bf16"},
        {"name": "combine_prompt", "op": "combine", "tokens": 8192, "topk": 8, "c": 2048, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A size spread evenly over its logarithm: odd, a power of two, or a multiple of 160."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.randrange(3)
    v = v | 1 if kind == 0 else 1 << int(round(math.log2(v))) if kind == 1 else v // 160 * 160
    return min(hi, max(lo, v))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "grouped", "grouped", "combine"])
    if op == "quantize":
        hb = rng.choice([1, 2, 16, 32, 64, 128, 256])
        c = hb * _log(rng, max(1, 64 // hb), 16384 // hb)
        gated = rng.random() < 0.4
        rows = min(_log(rng, 1, 16384), max(1, 8192 * 4096 // (c * (2 if gated else 1))))
        gather = rng.random() < 0.3
        return {"op": op, "rows": rows, "src": max(1, rows // 4) if gather else rows, "c": c, "hb": hb,
                "dtype": rng.choice(["bf16", "f16", "f32"]), "act": rng.choice(["silu", "gelu"]) if gated else "none",
                "gated": gated, "gather": gather, "codes": rng.choice(["f16", "f16", "i8"])}
    if op == "linear":
        k, n = _log(rng, 64, 16384), _log(rng, 64, 16384)
        rows = min(_log(rng, 1, 16384), max(1, 8192 * 4096 * 16384 // (k * n)))
        return {"op": op, "rows": rows, "k": k, "n": n, "codes": "i8" if rows <= 8 else rng.choice(["f16", "f16", "i8"]),
                "out": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5}
    if op == "grouped":
        experts = rng.choice([4, 8, 16, 32, 60, 64, 128])
        k, n = _log(rng, 128, 4096), _log(rng, 128, 4096)
        while experts * k * n > 64 * 2048 * 2048:
            k, n = max(128, k // 2 | 1), max(128, n // 2 | 1)
        rows = _log(rng, 1, 32768)
        active = min(rows, rng.randint(experts * 3 // 4, experts))
        return {"op": op, "rows": rows, "experts": experts, "active": active, "k": k, "n": n,
                "codes": "i8" if rows <= 8 else rng.choice(["f16", "f16", "i8"]),
                "out": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5}
    topk = rng.choice([1, 2, 4, 6, 8])
    c = _log(rng, 64, 8192)
    return {"op": op, "tokens": min(_log(rng, 1, 16384), 8192 * 8 * 2048 // (topk * c)), "topk": topk, "c": c,
            "dtype": rng.choice(["bf16", "f16", "f32"])}


def work(case):
    op = case["op"]
    if op == "quantize":
        rows, c = case["rows"], case["c"]
        values = case["src"] * c * (2 if case["gated"] else 1)
        return {"bytes": values * SIZE[case["dtype"]] + rows * c * SIZE[case["codes"]] + 4 * rows * (1 + case["gather"]),
                "flops": rows * c * (math.log2(case["hb"]) + 3 + (8 if case["gated"] else 0))}
    if op in ("linear", "grouped"):
        rows, k, n = case["rows"], case["k"], case["n"]
        held = case.get("active", 1)
        return {"bytes": held * n * (k + 4 + 4 * case["bias"]) + rows * (k * SIZE[case["codes"]] + 4)
                + rows * n * SIZE[case["out"]] + 4 * (case.get("experts", -1) + 1), "flops": 2 * rows * n * k}
    t, j, c = case["tokens"], case["topk"], case["c"]
    return {"bytes": t * (j + 1) * c * SIZE[case["dtype"]] + 8 * t * j, "flops": 2 * t * j * c}


# ------------------------------------------------------------------ inputs

def _codes(g, rows, k, kind):
    """Gaussian codes, each row's largest at 127 or a little below, as a per-token quantizer leaves them."""
    v = (torch.randn(rows, k, generator=g, device="cuda") * 34).round_().clamp_(-127, 127)
    return v.to(torch.int8 if kind == "i8" else torch.float16)


def _offsets(case, seed):
    """Ragged row counts: `active` experts hold a row at least, the rest of the rows by a skewed popularity."""
    r = np.random.RandomState(seed % (1 << 31))
    held = r.permutation(case["experts"])[: case["active"]]
    p = np.exp(r.standard_normal(case["active"]))
    counts = np.zeros(case["experts"], np.int64)
    counts[held] = 1 + r.multinomial(case["rows"] - case["active"], p / p.sum())
    return np.concatenate([[0], np.cumsum(counts)]), int(counts.max())


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, s = case["op"], dict(case)
    if op == "quantize":
        width = case["c"] * (2 if case["gated"] else 1)
        # a channel's own spread, and a few outlier channels, as activations have them
        spread = torch.exp(0.5 * torch.randn(width, generator=g, device="cuda"))
        spread[torch.randint(0, width, (4,), generator=g, device="cuda")] *= 20
        s["x"] = (torch.randn(case["src"], width, generator=g, device="cuda") * spread).to(DTYPES[case["dtype"]])
        s["index"] = None
        if case["gather"]:
            i = torch.randint(0, case["src"], (case["rows"],), generator=g, device="cuda")
            empty = torch.rand(case["rows"], generator=g, device="cuda") < 0.02
            s["index"] = torch.where(empty, -1, i).to(torch.int32)
        h = torch.ones(1, 1, device="cuda")
        while h.shape[0] < case["hb"]:
            h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
        s["h"] = h
        return s
    if op == "combine":
        t, j = case["tokens"], case["topk"]
        s["y"] = torch.randn(t * j, case["c"], generator=g, device="cuda").to(DTYPES[case["dtype"]])
        at = torch.randperm(t * j, generator=g, device="cuda").reshape(t, j)
        gone = torch.rand(t, j, generator=g, device="cuda") < 0.02          # slots over an expert's capacity
        s["index"] = torch.where(gone, -1, at).to(torch.int32)
        s["weights"] = torch.softmax(torch.randn(t, j, generator=g, device="cuda"), -1)
        return s
    rows, k, n, e = case["rows"], case["k"], case["n"], case.get("experts", 1)
    s["x"] = _codes(g, rows, k, case["codes"])
    s["sx"] = 0.02 * torch.exp(0.3 * torch.randn(rows, generator=g, device="cuda"))
    w = torch.empty(e, n, k, dtype=torch.int8, device="cuda")
    for i in range(e):
        w[i] = _codes(g, n, k, "i8")
    s["w"], s["sw"] = w, 0.001 * torch.exp(0.2 * torch.randn(e, n, generator=g, device="cuda"))
    s["b"] = torch.randn(e, n, generator=g, device="cuda") if case["bias"] else None
    if op == "grouped":
        off, s["most"] = _offsets(case, seed)
        s["offsets"] = torch.from_numpy(off).to(torch.int32).cuda()
    if own:
        from paper_2608_01653_gb300 import hatq
        one = op == "linear"
        s["layer"] = hatq.prepare_linear(w[0] if one else w, scales=s["sw"][0] if one else s["sw"],
                                         bias=s["b"] if s["b"] is None or not one else s["b"][0])
    return s


# ------------------------------------------------------------------ the operators

def _activation(v, act):
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5))) if act == "gelu" else v


def _quantize(s):
    x, c = s["x"], s["c"]
    if s["index"] is not None:
        i = s["index"].long()
        x = torch.where((i < 0)[:, None], 0, x[i.clamp(min=0)])
    x = x.float()
    x = _activation(x[:, :c], s["act"]) * x[:, c:] if s["gated"] else _activation(x, s["act"])
    t = (x.reshape(-1, s["hb"]) @ s["h"]).reshape(x.shape) if s["hb"] > 1 else x
    a = t.abs().amax(1, keepdim=True)
    codes = torch.where(a > 0, (t * (127 / a)).round().clamp(-127, 127), 0)
    scales = torch.where(a > 0, a / 127 / math.sqrt(s["hb"]), 1)[:, 0]
    # 16-bit codes are returned as they are, 8-bit ones as the values they stand for
    return (codes.half(), scales) if s["codes"] == "f16" else (codes * scales[:, None], scales)


def _linear(s):
    y = (s["x"].float() @ s["w"][0].float().T) * s["sw"] * s["sx"][:, None]
    return (y if s["b"] is None else y + s["b"]).to(DTYPES[s["out"]])


def _grouped(s):
    x, w, off = s["x"].float(), s["w"], s["offsets"].long()
    r = torch.arange(s["rows"], device=x.device)
    e = torch.searchsorted(off, r, right=True) - 1
    if s["rows"] <= s["active"]:                     # a row or so each: the row's own matrix
        y = torch.bmm(w[e].float(), x[:, :, None])[:, :, 0]
    else:                                            # the experts' rows, padded to the longest
        padded = x.new_zeros(s["experts"], s["most"], s["k"])
        padded[e, r - off[e]] = x
        y = torch.bmm(padded, w.float().transpose(1, 2))[e, r - off[e]]
    y = y * s["sw"][e] * s["sx"][:, None]
    return (y if s["b"] is None else y + s["b"][e]).to(DTYPES[s["out"]])


def _combine(s):
    i = s["index"].long()
    z = torch.where((i < 0)[:, :, None], 0, s["y"].float()[i.clamp(min=0)])
    return (z * s["weights"][:, :, None]).sum(1).to(DTYPES[s["dtype"]])


def run(s):
    op = s["op"]
    if not own:
        return {"quantize": _quantize, "linear": _linear, "grouped": _grouped, "combine": _combine}[op](s)
    from paper_2608_01653_gb300 import hatq
    if op == "quantize":
        codes, scales = hatq.quantize_tokens(s["x"], hb=s["hb"], act=s["act"], gated=s["gated"], rows=s["index"],
                                             codes=s["codes"])
        return (codes, scales) if s["codes"] == "f16" else (codes * scales[:, None], scales)
    if op == "linear":
        return hatq.linear(s["x"], s["sx"], s["layer"], dtype=DTYPES[s["out"]])
    if op == "grouped":
        return hatq.grouped_linear(s["x"], s["sx"], s["offsets"], s["layer"], dtype=DTYPES[s["out"]])
    return hatq.combine_rows(s["y"], s["index"], s["weights"])


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] == "quantize":
        x = s["x"].to(d)
        if s["index"] is not None:
            source = torch.cat([x, x.new_zeros(1, x.shape[1])])
            x = source[torch.where(s["index"] < 0, case["src"], s["index"]).long()]
        if case["gated"]:
            gate, up = x.chunk(2, 1)
            x = up * (torch.nn.functional.silu(gate) if case["act"] == "silu" else torch.nn.functional.gelu(gate))
        hb, i = case["hb"], np.arange(case["hb"])
        parity = np.array([[bin(a & b).count("1") & 1 for b in i] for a in i])
        hadamard = torch.from_numpy(1.0 - 2.0 * parity).to(x) / math.sqrt(hb)
        t = torch.einsum("rbi,ij->rbj", x.reshape(x.shape[0], -1, hb), hadamard).reshape(x.shape)
        step = t.abs().amax(1) / 127
        step[step == 0] = 1
        codes = torch.round(t / step[:, None])
        return (codes if case["codes"] == "f16" else codes * step[:, None]), step
    if case["op"] == "combine":
        y = torch.cat([s["y"].to(d), s["y"].new_zeros(1, case["c"], dtype=d)])
        out = y.new_zeros(case["tokens"], case["c"])
        for j in range(case["topk"]):
            at = torch.where(s["index"][:, j] < 0, case["tokens"] * case["topk"], s["index"][:, j]).long()
            out += s["weights"][:, j].to(d)[:, None] * y[at]
        return out
    out = torch.empty(case["rows"], case["n"], dtype=d, device="cuda")
    off = s["offsets"].tolist() if case["op"] == "grouped" else [0, case["rows"]]
    if 2 * case["rows"] * case["n"] * case["k"] > 1.2e13:
        return None
    for e in range(len(off) - 1):
        at = slice(off[e], off[e + 1])
        if off[e] < off[e + 1]:
            out[at] = (s["x"][at].to(d) @ s["w"][e].to(d).T) * s["sw"][e].to(d) * s["sx"][at].to(d)[:, None]
            if s["b"] is not None:
                out[at] += s["b"][e].to(d)
    return out
