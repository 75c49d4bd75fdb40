"""Operators of the inference-time cache as measurable cases: attention that accumulates the weights its rows receive,
eviction by those weights, and the same over a cache that is held in 8 bits with a scale per block of rows and KV head.

Where `own` is false, `run` computes an operator from elementary torch operations in 32 bits; where it is true it makes
the library's call.  `exact` is the definition in 64 bits, written apart from both.

Shapes: B sequences, Hq / Hkv query and KV heads, d channels, n rows of the longest sequence.  `ragged`: the other
sequences are shorter (see _lengths); the cache has room for more rows than n, as a serving cache has.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMATS = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"int8": 127.0, "e4m3": 448.0}       # the largest code of a format
LEAST = -120                               # the least exponent of a scale


def _case(kind, name, B, Hq, Hkv, d, n, dtype="bf16", **more):
    return dict(name=name, kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, n=n, dtype=dtype, **more)


def listed():
    return [
        # ---- a new token attends over the cache, and every row is credited with the weight it received ----
        # a small model in single precision, short histories: launches and latency
        _case("attend", "attend_short_f32", 2, 16, 4, 64, 777, "f32", decay=1.0),
        # eight requests with a long history each
        _case("attend", "attend_16k_b8", 8, 32, 8, 128, 16401, decay=0.99),
        # ---- the cache has outgrown its budget: the rows with the least weight go ----
        # one request, halved
        _case("evict", "evict_4k", 1, 32, 8, 128, 4501, S=4, recent=256, budget=2048),
        # four requests of 32K tokens, a quarter kept
        _case("evict", "evict_32k_b4", 4, 32, 8, 128, 32768, S=64, recent=1024, budget=8192),
        # ---- rows go into the 8-bit cache, and the blocks that they touch are read back ----
        # one token for each of sixteen requests, in part-filled blocks
        _case("append", "append_token_b16", 16, 32, 8, 128, 4093, format="int8", block=64, T=1, ragged=True),
        # the K and V of a long prompt
        _case("append", "append_prompt_32k", 1, 32, 8, 128, 0, format="e4m3", block=64, T=32001, ragged=False),
        # ---- attention over the 8-bit cache ----
        # one token of one request with a short history of no round length: latency
        _case("attend_quant", "quant_short", 1, 12, 2, 128, 777, format="int8", block=64, T=1, ragged=False, acc=False, decay=1.0),
        # eight requests of different lengths up to 32K, the weights accumulated for a later eviction
        _case("attend_quant", "quant_32k_b8", 8, 32, 8, 128, 32768, format="int8", block=64, T=1, ragged=True, acc=True, decay=1.0),
        # the longest context in use, many query heads
        _case("attend_quant", "quant_128k", 1, 64, 8, 128, 131072, format="e4m3", block=128, T=1, ragged=False, acc=False, decay=1.0),
        # five drafted tokens of each request at once, single precision, head_dim 64
        _case("attend_quant", "quant_tokens_f32", 4, 16, 4, 64, 8191, "f32", format="e4m3", block=32, T=5, ragged=True, acc=True, decay=1.0),
        # ---- eviction on the 8-bit cache (rows change their blocks, blocks their scales), the kept rows read back ----
        # two short requests of a small model
        _case("evict_quant", "evict_quant_8k", 2, 12, 2, 128, 8111, format="int8", block=64, S=4, recent=256, budget=2048, ragged=False),
        # eight requests of up to 32K tokens, a quarter kept
        _case("evict_quant", "evict_quant_32k_b8", 8, 32, 8, 128, 32768, format="e4m3", block=64, S=64, recent=1024, budget=8192, ragged=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the ranges above; lengths are mostly of no round size."""
    kind = rng.choice(["attend", "attend", "evict", "evict", "append", "attend_quant", "attend_quant", "attend_quant", "evict_quant"])
    dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
    Hkv, G = rng.choice([1, 2, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 6, 8])
    c = dict(kind=kind, Hq=Hkv * G, Hkv=Hkv, d=d, dtype=dtype)
    n = _logint(rng, 200, 33000)
    B = rng.choice([1, 1, 2, 4, 8]) if n > 8000 else rng.choice([1, 2, 3, 8, 16])
    quant = dict(format=rng.choice(["int8", "e4m3"]), block=rng.choice([16, 32, 64, 64, 128]), ragged=rng.random() < 0.6)
    keep = dict(S=rng.choice([0, 4, 16, 33, 64]), recent=_logint(rng, 16, 64 + n // 16))
    keep["budget"] = min(n, max(keep["S"] + keep["recent"] + 1, int(n * rng.choice([0.125, 0.25, 0.5, 0.75])) + rng.randint(0, 40)))
    if kind == "attend":
        return dict(c, B=min(B, (2 if n > 16000 else 4) if dtype == "f32" else 4 if n > 16000 else 8), n=n, decay=rng.choice([1.0, 1.0, 0.98]))
    if kind == "evict":
        return dict(c, B=min(B, 1 if dtype == "f32" else 2) if n > 8000 else min(B, 4), n=n, **keep)
    if kind == "append":
        if rng.random() < 0.5:
            return dict(c, B=B, n=n // 4, T=rng.choice([1, 1, 2, 7, 16]), **quant)
        return dict(c, B=1 if n > 8000 else 2, n=rng.choice([0, n // 3]), T=min(n, 24000) if dtype == "f32" else n, **quant)
    if kind == "attend_quant":
        return dict(c, B=B, n=n, T=rng.choice([1, 1, 1, 1, 2, 4, 9]) if n * B * Hkv < 1 << 20 else 1, acc=rng.random() < 0.5, decay=1.0, **quant)
    return dict(c, B=min(B, 2) if n > 8000 else min(B, 8), n=n, **keep, **quant)


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(c):
    """Rows of every sequence: the first has n, the others of a ragged batch down to a third of it."""
    B, n = c["B"], c["n"]
    return [n - (b * n * 2) // (3 * B) if c.get("ragged") else n for b in range(B)]


def _cap(c):
    """Rows that the cache has room for: whole blocks, some more than are there or come."""
    return (c["n"] + c.get("T", 1) + 64 + 127) // 128 * 128


def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _rows(g, which, shape, dtype):
    """Rows as attention layers make them: channels of unequal size, K with four large ones per head and some rows larger."""
    B, H, n, d = shape
    x = _normal(g, shape)
    x *= 0.5 + torch.rand((1, H, 1, d), generator=g, device=DEV)
    if which == "K":
        ch = torch.rand((1, H, 1, d), generator=g, device=DEV).argsort(-1)
        x *= torch.where(ch < 4, 4.0, 1.0)
    x *= torch.where(torch.rand((B, H, n, 1), generator=g, device=DEV) < 0.01, 3.0, 1.0)
    return x.to(dtype)


def _weights(g, shape):
    """Accumulated weights: a heavy tail, and rows that never received any."""
    return _normal(g, shape).mul_(2).exp_() * (torch.rand(shape, generator=g, device=DEV) > 0.1)


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    B, Hq, Hkv, d, n, cap = c["B"], c["Hq"], c["Hkv"], c["d"], c["n"], _cap(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, s = c["kind"], {"case": case, "cap": cap}
    lens = _lengths(c)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if kind in ("attend", "evict"):
        for z in ("K", "V"):
            s[z] = _rows(g, z, (B, Hkv, cap, d), dt)
    else:
        for z in ("K", "V"):
            x = _rows(g, z, (B, Hkv, cap, d), torch.float32)
            s[z + "c"], s[z + "s"] = _to_codes(x.view(B, Hkv, cap // c["block"], c["block"], d), c["format"])
            s[z + "c"] = s[z + "c"].view(B, Hkv, cap, d)
            del x
    if kind in ("attend", "attend_quant"):
        s["q"] = _normal(g, (B, Hq, d) if kind == "attend" else (B, Hq, c["T"], d), dt)
        s["O"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:-1], dtype=torch.float32, device=DEV)
        if c.get("acc", True):
            s["acc"] = _weights(g, (B, Hkv, cap)) * (Hq // Hkv / n)         # of a few tokens before this one
            s["acc_out"] = torch.zeros_like(s["acc"])
    if kind == "append":
        T = c["T"]
        for z in ("K", "V"):
            s[z + "new"] = _rows(g, z, (B, Hkv, T, d), dt)
        s["first"] = s["lens"] // c["block"] * c["block"]
        s["after"] = s["lens"] + T
        s["window"] = max(-(-(a + T) // c["block"]) - a // c["block"] for a in lens) * c["block"]
        for z in ("K", "V"):
            s[z + "r"] = torch.empty((B, Hkv, s["window"], d), dtype=dt, device=DEV)
    if kind in ("evict", "evict_quant"):
        s["acc"] = _weights(g, (B, Hkv, cap))
        s["pos"] = torch.arange(cap, dtype=torch.int32, device=DEV).expand(B, Hkv, cap).contiguous()
        s["acc_o"] = torch.empty_like(s["acc"])
        s["pos_o"] = torch.full_like(s["pos"], -1)
        s["lens_o"] = torch.zeros_like(s["lens"])
        for z in ("K", "V"):
            if kind == "evict":
                s[z + "o"] = torch.zeros_like(s[z])
            else:
                s[z + "co"], s[z + "so"] = torch.zeros_like(s[z + "c"]), torch.zeros_like(s[z + "s"])
                s[z + "r"] = torch.empty((B, Hkv, c["budget"], d), dtype=dt, device=DEV)
    if own:
        _handles(s)       # the parameters, cache objects and workspace that a program keeps
    return s


def _handles(s):
    import paper_2506_11498_amd as lrsa
    c, cap = s["case"], s["cap"]
    B, Hq, Hkv, d, kind = c["B"], c["Hq"], c["Hkv"], c["d"], c["kind"]
    rows = s["K"] if "K" in s else s["Knew"] if "Knew" in s else s["Kr"] if "Kr" in s else torch.empty((B, Hkv, 1, d), dtype=DTYPES[c["dtype"]], device=DEV)
    s["p"] = lrsa.make_params((B, Hq, cap, d), (B, Hkv, cap, d), (Hq * cap * d, cap * d, d, 1), rows.stride(), dtype=DTYPES[c["dtype"]],
                              sink=c.get("S", 0), lag=64, topk=16)
    if "Kc" in s:
        s["cache"] = lrsa.QuantCache(s["Kc"], s["Vc"], s["Ks"], s["Vs"], c["block"])
    if "Kco" in s:
        s["cache_o"] = lrsa.QuantCache(s["Kco"], s["Vco"], s["Kso"], s["Vso"], c["block"])
    if "Kr" in s:
        s["pr"] = lrsa.make_params((B, Hq, cap, d), (B, Hkv, cap, d), (Hq * cap * d, cap * d, d, 1), s["Kr"].stride(), dtype=DTYPES[c["dtype"]],
                                   sink=c.get("S", 0), lag=64, topk=16)
    need = {"attend": lambda: lrsa.decode_attn_acc_ws_bytes(s["p"], c["n"]),
            "evict": lambda: lrsa.cache_evict_ws_bytes(s["p"], c["n"], c["budget"]),
            "append": lambda: 0,
            "attend_quant": lambda: lrsa.decode_attn_quant_ws_bytes(s["p"], c["T"], c["n"], c["acc"]),
            "evict_quant": lambda: lrsa.cache_evict_ws_bytes(s["p"], c["n"], c["budget"])}[kind]()
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------------ one pass: the library's calls
def _run_own(s):
    import paper_2506_11498_amd as lrsa
    c, p = s["case"], s["p"]
    kind, n = c["kind"], c["n"]
    if kind == "attend":
        lrsa.lrsa_decode_attn_acc(p, s["q"], s["K"], s["V"], n, s["acc"], s["acc_out"], c["decay"], s["O"], s["lse"], s["ws"])
        return {"O": s["O"], "lse": s["lse"], "acc": s["acc_out"]}
    if kind == "evict":
        new = lrsa.lrsa_cache_evict(p, s["K"], s["V"], s["pos"], s["acc"], n, c["budget"], c["recent"], s["Ko"], s["Vo"], s["pos_o"], s["acc_o"], s["ws"])
        return {"K": s["Ko"][:, :, :new], "V": s["Vo"][:, :, :new], "pos": s["pos_o"], "acc": s["acc_o"], "length": new}
    if kind == "append":
        lrsa.lrsa_cache_append_quant(p, s["cache"], s["Knew"], s["Vnew"], s["lens"])
        lrsa.lrsa_cache_read_quant(s["pr"], s["cache"], s["after"], s["window"], s["first"], s["Kr"], s["Vr"])
        return {"K": s["Kr"], "V": s["Vr"]}
    if kind == "attend_quant":
        lrsa.lrsa_decode_attn_quant(p, s["q"], s["cache"], s["lens"], n, s.get("acc"), s.get("acc_out"), c["decay"], s["O"], s["lse"], s["ws"])
        return {"O": s["O"], "lse": s["lse"], **({"acc": s["acc_out"]} if c["acc"] else {})}
    lrsa.lrsa_cache_evict_quant(p, s["cache"], s["pos"], s["acc"], s["lens"], n, c["budget"], c["recent"], s["cache_o"], s["pos_o"], s["acc_o"], s["lens_o"], s["ws"])
    lrsa.lrsa_cache_read_quant(s["pr"], s["cache_o"], s["lens_o"], c["budget"], None, s["Kr"], s["Vr"])
    return {"K": s["Kr"], "V": s["Vr"], "pos": s["pos_o"], "acc": s["acc_o"], "lens": s["lens_o"]}


# ------------------------------------------------------------------------------------------------ one pass: plain forms
def _two_to(e):
    """2^e as the 32-bit number with that exponent field."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale_of(top, fmt):
    """The smallest power of two by which `top` (a largest magnitude) does not exceed the largest code."""
    m, e = torch.frexp(top)                                     # top = m 2^e, 1/2 <= m < 1
    lim, up = (TOP[fmt] / 128, 7) if fmt == "int8" else (TOP[fmt] / 512, 9)
    e = torch.where(top == 0, LEAST, (e - up + (m > lim).int())).clamp(min=LEAST)
    return _two_to(e)


def _round_codes(y, fmt):
    """The nearest code, ties to even, as a 32-bit value."""
    if fmt == "int8":
        return y.round().clamp(-127, 127)
    step = _two_to((torch.frexp(y)[1] - 4).clamp(min=-9))      # of e4m3: 3 bits behind the point, subnormals below 2^-6
    return (y / step).round().mul_(step).clamp_(-448, 448)


def _to_codes(x, fmt):
    """Blocks x [..., rows, d] -> codes, scales [...]."""
    s = _scale_of(x.abs().amax((-2, -1)), fmt)
    return _round_codes(x / s[..., None, None], fmt).to(FORMATS[fmt]), s


def _values(codes, scales, block, n):
    """The first n rows of a cache as 32-bit values."""
    B, H, cap, d = codes.shape
    nb = -(-n // block)
    x = codes[:, :, :nb * block].to(torch.float32).view(B, H, nb, block, d) * scales[:, :, :nb, None, None]
    return x.view(B, H, nb * block, d)[:, :, :n]


def _attend(q, K, V, lens, decay, acc, acc_out, dt):
    """q [B, Hq, T, d], K and V [B, Hkv, n, d] in 32 bits; token t of T sees rows before lens - T + 1 + t."""
    B, Hq, T, d = q.shape
    Hkv, n = K.shape[1:3]
    s = torch.matmul(q.to(torch.float32).view(B, Hkv, Hq // Hkv * T, d), K.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(B, Hkv, Hq // Hkv, T, n)
    seen = torch.arange(n, device=DEV) < (lens[:, None] - T + 1 + torch.arange(T, device=DEV))[:, :, None]      # [B, T, n]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    lse = (total.log() + top).view(B, Hq, T)
    s.div_(torch.where(total == 0, 1.0, total))
    O = torch.matmul(s.view(B, Hkv, Hq // Hkv * T, n), V).view(B, Hq, T, d).to(dt)
    if acc is None:
        return O, lse, None
    there = torch.arange(n, device=DEV) < lens[:, None, None]
    out = acc_out.clone()
    out[:, :, :n] = torch.where(there, decay * acc[:, :, :n] + s.sum((2, 3)), out[:, :, :n])
    return O, lse, out


def _kept(acc, lens, S, recent, budget):
    """Rows that stay, in order: [B, Hkv, budget] with garbage behind the new lengths; the new lengths [B]."""
    r, n = torch.arange(acc.shape[-1], device=DEV), lens[:, None, None]
    key = torch.where((r < S) | (r >= n - recent), math.inf, acc)
    key = torch.where(r < n, key, -math.inf)
    first = key.argsort(dim=-1, descending=True, stable=True)[..., :budget]      # ties: the lowest row first
    new = lens.clamp(max=budget)
    first = torch.where(torch.arange(budget, device=DEV) < new[:, None, None], first, acc.shape[-1] - 1)
    return first.sort(-1).values, new


def _evict_rows(s, x, kept):
    return x.gather(2, kept[..., None].expand(*kept.shape, x.shape[-1]))


def _evict_lists(s, kept, new):
    budget = kept.shape[-1]
    there = torch.arange(budget, device=DEV) < new[:, None, None]
    pos, acc = s["pos_o"].clone(), torch.zeros_like(s["acc"])
    pos[:, :, :budget] = torch.where(there, s["pos"].gather(2, kept), pos[:, :, :budget])
    acc[:, :, :budget] = torch.where(there, s["acc"].gather(2, kept), 0.0)
    return pos, acc, there


def _run_plain(s):
    c = s["case"]
    kind, n, dt, fmt, block = c["kind"], c["n"], DTYPES[c["dtype"]], c.get("format"), c.get("block")
    if kind == "attend":
        q = s["q"][:, :, None]
        O, lse, acc = _attend(q, s["K"][:, :, :n].to(torch.float32), s["V"][:, :, :n].to(torch.float32), s["lens"], c["decay"], s["acc"], s["acc_out"], dt)
        return {"O": O[:, :, 0], "lse": lse[:, :, 0], "acc": acc}
    if kind == "attend_quant":
        K, V = (_values(s[z + "c"], s[z + "s"], block, n) for z in ("K", "V"))
        O, lse, acc = _attend(s["q"], K, V, s["lens"], c["decay"], s.get("acc"), s.get("acc_out"), dt)
        return {"O": O, "lse": lse, **({"acc": acc} if c["acc"] else {})}
    if kind == "append":
        return {z: _append_plain(s, z) for z in ("K", "V")}
    if kind == "evict":
        kept, new = _kept(s["acc"], s["lens"], c["S"], c["recent"], c["budget"])
        rows = min(n, c["budget"])
        pos, acc, _ = _evict_lists(s, kept, new)
        return {"K": _evict_rows(s, s["K"], kept[:, :, :rows]), "V": _evict_rows(s, s["V"], kept[:, :, :rows]), "pos": pos, "acc": acc, "length": rows}
    kept, new = _kept(s["acc"], s["lens"], c["S"], c["recent"], c["budget"])
    pos, acc, there = _evict_lists(s, kept, new)
    return {**{z: _evict_values(s, z, kept, there) for z in ("K", "V")}, "pos": pos, "acc": acc, "lens": new}


def _evict_values(s, z, kept, there):
    c, d = s["case"], s["case"]["d"]
    B, H, budget = kept.shape
    block, nb = c["block"], -(-budget // c["block"])
    x = _evict_rows(s, s[z + "c"].view(torch.uint8), kept).view(FORMATS[c["format"]]).to(torch.float32)
    x = torch.where(there[..., None], x * s[z + "s"].gather(2, kept // block)[..., None], 0.0)
    blocks = torch.zeros((B, H, nb * block, d), device=DEV)
    blocks[:, :, :budget] = x
    blocks = blocks.view(B, H, nb, block, d)
    scale = _scale_of(blocks.abs().amax((-2, -1)), c["format"])[..., None, None]
    return _round_codes(blocks / scale, c["format"]).mul_(scale).view(B, H, nb * block, d)[:, :, :budget].to(DTYPES[c["dtype"]])


def _append_plain(s, z):
    """The blocks that new rows touch, as values after the call; zero behind the last row."""
    c = s["case"]
    B, H, d, T, fmt, block = c["B"], c["Hkv"], c["d"], c["T"], c["format"], c["block"]
    lens, W = s["lens"], s["window"]
    r = s["first"][:, None] + torch.arange(W, device=DEV)                        # cache rows of the window [B, W]
    older, newer = r < lens[:, None], (r >= lens[:, None]) & (r < s["after"][:, None])
    at = (r - lens[:, None]).clamp(0, T - 1)[:, None, :, None].expand(B, H, W, d)
    x = torch.where(newer[:, None, :, None], s[z + "new"].gather(2, at).to(torch.float32), 0.0).view(B, H, W // block, block, d)
    scale = _scale_of(x.abs().amax((-2, -1)), fmt)
    # the first block may hold older rows: its scale is kept where it is large enough, and its codes change with the scale
    j = (s["first"] // block)[:, None, None].expand(B, H, 1)
    before = torch.where((lens > s["first"])[:, None, None], s[z + "s"].gather(2, j.long()), 0.0)
    scale[:, :, :1] = torch.maximum(scale[:, :, :1], before)
    out = _round_codes(x / scale[..., None, None], fmt).mul_(scale[..., None, None]).view(B, H, W, d)
    rows = r[:, :block].clamp(max=s["cap"] - 1)[:, None, :, None].expand(B, H, block, d)
    codes = s[z + "c"].view(torch.uint8).gather(2, rows.long()).view(FORMATS[fmt]).to(torch.float32)
    now = scale[:, :, :1, None]
    codes = _round_codes(codes * (before[..., None] / now), fmt) * now
    out[:, :, :block] = torch.where(older[:, None, :block, None], codes, out[:, :, :block])
    return out.to(DTYPES[c["dtype"]])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _code_values(fmt):
    """Every value that a code stands for, ascending; of e4m3 the 8 bits are sign, exponent (bias 7), 3 bits of fraction."""
    if fmt == "int8":
        return np.arange(-127, 128, dtype=np.float64)
    b = np.arange(127)                       # 127 is no number
    e, f = b >> 3, b & 7
    v = np.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (e - 7.0))
    return np.concatenate([-v[:0:-1], v])


def _nearest(y, fmt):
    """y (64 bits, CUDA) -> the nearest of the code values, a tie to the one with an even code."""
    t = torch.from_numpy(_code_values(fmt)).to(y.device)
    mid = (t[1:] + t[:-1]) / 2
    i = torch.bucketize(y, mid)              # the first mid >= y: a tie goes to the lower value ...
    tie = (i < len(mid)) & (y == mid[i.clamp(max=len(mid) - 1)])
    zero = len(t) // 2
    return t[i + (tie & ((i - zero) % 2 != 0))]      # ... unless that one's code is odd


def _pow2(top, fmt):
    """The first of the powers of two from 2^LEAST on that is large enough."""
    powers = torch.tensor([2.0 ** e for e in range(LEAST, 130)], dtype=torch.float64, device=top.device)
    return powers[torch.bucketize(top, powers * TOP[fmt])]


def _cache64(s, z, b, h, rows):
    """Rows of a cache of 8 bits, or of one that holds values."""
    if z in s:
        return s[z][b, h, rows].double()
    return s[z + "c"].view(torch.uint8)[b, h, rows].view(s[z + "c"].dtype).double() * s[z + "s"][b, h].double()[rows // s["case"]["block"]][:, None]


def _exact_attend(s):
    c, n = s["case"], s["case"]["n"]
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    T, G = c.get("T", 1), Hq // Hkv
    q = s["q"].double().view(B, Hq, T, d)
    O = torch.zeros((B, Hq, T, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
    acc = s["acc_out"].double() if "acc_out" in s else None
    for b, length in enumerate(_lengths(c)):
        for h in range(Hkv):
            rows = torch.arange(length, device=DEV)
            K, V = (_cache64(s, z, b, h, rows) for z in ("K", "V"))
            w_rows = torch.zeros(length, dtype=torch.float64, device=DEV)
            for t in range(T):
                m = length - T + 1 + t
                if m <= 0:
                    continue
                heads = slice(h * G, (h + 1) * G)
                x = q[b, heads, t] @ K[:m].T / d ** 0.5
                lse[b, heads, t] = torch.logsumexp(x, -1)
                w = torch.softmax(x, -1)
                O[b, heads, t] = w @ V[:m]
                w_rows[:m] += w.sum(0)
            if acc is not None:
                acc[b, h, :length] = c["decay"] * s["acc"][b, h, :length].double() + w_rows
    O, lse = (O[:, :, 0], lse[:, :, 0]) if c["kind"] == "attend" else (O, lse)
    return {"O": O, "lse": lse, **({"acc": acc} if acc is not None else {})}


def _exact_rows(s, b, h, length):
    """The surviving rows of one head, by their weights as numbers of 64 bits."""
    c = s["case"]
    if length <= c["budget"]:
        return np.arange(length)
    a = s["acc"][b, h, :length].double().cpu().numpy()
    lo, hi = c["S"], length - c["recent"]
    best = lo + np.lexsort((np.arange(hi - lo), -a[lo:hi]))[:c["budget"] - c["S"] - c["recent"]]
    return np.concatenate([np.arange(lo), np.sort(best), np.arange(hi, length)])


def _exact_evict(s):
    c, B, Hkv, d, cap = s["case"], s["case"]["B"], s["case"]["Hkv"], s["case"]["d"], s["cap"]
    quant, lens = c["kind"] == "evict_quant", _lengths(c)
    new = [min(x, c["budget"]) for x in lens]
    width = c["budget"] if quant else new[0]
    out = {z: torch.zeros((B, Hkv, width, d), dtype=torch.float64, device=DEV) for z in ("K", "V")}
    pos, acc = s["pos_o"].clone(), torch.zeros((B, Hkv, cap), dtype=torch.float64, device=DEV)
    for b in range(B):
        for h in range(Hkv):
            rows = torch.from_numpy(_exact_rows(s, b, h, lens[b])).to(DEV)
            pos[b, h, :new[b]] = s["pos"][b, h, rows]
            acc[b, h, :new[b]] = s["acc"][b, h, rows].double()
            for z in ("K", "V"):
                x = _cache64(s, z, b, h, rows)
                if quant:
                    k = c["block"]
                    full = torch.zeros((-(-new[b] // k) * k, d), dtype=torch.float64, device=DEV)
                    full[:new[b]] = x
                    full = full.view(-1, k * d)
                    scale = _pow2(full.abs().amax(1), c["format"])[:, None]
                    x = (_nearest(full / scale, c["format"]) * scale).view(-1, d)[:new[b]]
                out[z][b, h, :new[b]] = x
    return {**out, "pos": pos, "acc": acc, **({"lens": torch.tensor(new, dtype=torch.int32)} if quant else {"length": new[0]})}


def _exact_append(s):
    c, W, cap = s["case"], s["window"], s["cap"]
    B, Hkv, d, T, k, fmt = c["B"], c["Hkv"], c["d"], c["T"], c["block"], c["format"]
    out = {}
    for z in ("K", "V"):
        y = out[z] = torch.zeros((B, Hkv, W, d), dtype=torch.float64, device=DEV)
        for b, length in enumerate(_lengths(c)):
            first, left = length // k * k, length % k
            for h in range(Hkv):
                x = s[z + "new"][b, h].double()
                if left:                     # into the part-filled block
                    before = s[z + "s"][b, h, first // k].double()
                    part = x[:k - left]
                    scale = torch.maximum(_pow2(part.abs().amax(), fmt), before)
                    old = _cache64(s, z, b, h, torch.arange(first, length, device=DEV))
                    y[b, h, :left] = _nearest(old / scale, fmt) * scale
                    y[b, h, left:left + len(part)] = _nearest(part / scale, fmt) * scale
                    x = x[k - left:]
                if len(x):
                    full = torch.zeros((-(-len(x) // k) * k, d), dtype=torch.float64, device=DEV)
                    full[:len(x)] = x
                    full = full.view(-1, k * d)
                    scale = _pow2(full.abs().amax(1), fmt)[:, None]
                    at = k if left else 0
                    y[b, h, at:at + len(x)] = (_nearest(full / scale, fmt) * scale).view(-1, d)[:len(x)]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return _exact_append(s) if kind == "append" else _exact_evict(s) if kind in ("evict", "evict_quant") else _exact_attend(s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    B, Hq, Hkv, d, n, kind = c["B"], c["Hq"], c["Hkv"], c["d"], c["n"], c["kind"]
    rows = sum(_lengths(c)) * Hkv                                # rows of all sequences and KV heads
    if kind == "attend":
        return {"bytes": rows * (2 * d * e + 8) + B * Hq * (2 * d * e + 4), "flops": 4.0 * rows * Hq // Hkv * d}
    if kind == "attend_quant":
        scales = 2 * 4 * rows / c["block"]
        return {"bytes": rows * (2 * d + (8 if c["acc"] else 0)) + scales + B * Hq * c["T"] * (2 * d * e + 4), "flops": 4.0 * rows * Hq // Hkv * c["T"] * d}
    if kind == "append":
        new = B * Hkv * c["T"] * 2 * d                           # values in, codes out; the blocks' codes in, values out
        back = B * Hkv * 2 * d * sum(x % c["block"] + c["T"] for x in _lengths(c)) / B
        return {"bytes": new * (e + 1) + back * (1 + e), "flops": 2.0 * (new + back)}
    kept = sum(min(x, c["budget"]) for x in _lengths(c)) * Hkv
    lists = rows * 4 + kept * (4 + 8) + B * Hkv * _cap(c) * 4    # weights in; positions and weights out
    if kind == "evict":
        return {"bytes": kept * 2 * 2 * d * e + lists, "flops": 1.0 * rows}
    return {"bytes": kept * 2 * d * (2 + 1 + e) + lists, "flops": 2.0 * kept * 2 * d}
