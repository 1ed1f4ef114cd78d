"""Operators for repaired contexts that are kept in 8 bits, as measurable cases.

A repaired context, and the position-independent chunks that contexts are put together from, are kept longer than a request lasts.
In 8 bits with a power of two per token and head they take half the memory and half the time to read.  Four kinds of pass:

  rotate   norm of the query and key heads and rotary embedding in any of its forms: half or interleaved pairs, a part of the head,
           frequencies scaled for long contexts (`relaxkv_qk_norm_rotate`)
  write    norm, rotation and 8-bit append of K and V to a paged store, and the rows read back as the values they stand for
           (`relaxkv_append_quantized`, `relaxkv_read_quantized`)
  read     rows of the store back in bf16, their keys turned to another position (`relaxkv_read_quantized`)
  attend   attention of one or more new tokens of each sequence over its tokens in the store (`relaxkv_quantized_attention`)

Where `own` is false the same results come from elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# head geometries of this repository's workloads: the two model shapes of the benchmark, the decode tests' small model, the tiny one
LLAMA8B = dict(heads=32, kv_heads=8, head_dim=128)
QWEN14B = dict(heads=40, kv_heads=8, head_dim=128)
SMALL = dict(heads=8, kv_heads=2, head_dim=128)
TINY = dict(heads=4, kv_heads=1, head_dim=64)
RAGGED_CTX = (8192, 12288, 16384, 24576, 32768, 40960, 49152, 65536)      # the benchmark's ragged batch
TYPES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


def _text(xs):
    return ",".join(str(int(x)) for x in xs)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _rotate(geometry, rows, pairs, part, scaling, norm, **kw):
    """pairs: "half" or "interleaved"; part: dims of the head that are rotated."""
    return dict(kind="rotate", rows=rows, pairs=pairs, part=part, scaling=scaling, norm=norm, **geometry, **kw)


def _write(geometry, rows, block, type, pairs, part, scaling, norm, layout="token", **kw):
    """pairs "none": K and V as they are, out of a cache that is laid out like the store."""
    return dict(kind="write", rows=rows, block=block, type=type, pairs=pairs, part=part, scaling=scaling, norm=norm, layout=layout, **geometry, **kw)


def _read(geometry, rows, block, type, pairs, part, scaling, layout="token", **kw):
    return dict(kind="read", rows=rows, block=block, type=type, pairs=pairs, part=part, scaling=scaling, layout=layout, **geometry, **kw)


def _attend(geometry, lens, new, block, type, layout="token", **kw):
    """lens: tokens of each sequence, the `new` rows that attend among them."""
    return dict(kind="attend", lens=_text(lens), new=new, block=block, type=type, layout=layout, **geometry, **kw)


def _spread_lens(n, most, seed):
    rng = random.Random(seed)
    return [rng.randint(max(1, most // 16), most) for _ in range(n)]


def listed():
    return [
        # one decode step's rows of one layer; frequencies in bands, as models stretched to 128 K have them
        _rotate(LLAMA8B, 64, "half", 128, "bands", False, name="rotate_decode"),
        # the rows of a long prompt chunk: interleaved pairs of half the head, head norms, a ramp of scaled frequencies
        _rotate(QWEN14B, 8205, "interleaved", 64, "ramp", True, name="rotate_chunk"),
        # one decode step of 64 sequences appended in 8 bits
        _write(LLAMA8B, 64, 16, "int8", "half", 128, "bands", False, name="write_decode"),
        # a repaired context of 16 K tokens taken over from its bf16 cache, both head-major
        _write(QWEN14B, 16384, 64, "e4m3", "none", 0, "none", False, "head", name="write_context"),
        # a chunk of 512 tokens placed at another offset than the one it was encoded at
        _read(LLAMA8B, 512, 16, "int8", "half", 128, "bands", name="read_chunk"),
        # all chunks of a long, odd-sized context at once
        _read(QWEN14B, 32768 - 37, 64, "e4m3", "interleaved", 64, "linear", "head", name="read_context"),
        # the smallest attention call: one sequence of 1 K
        _attend(TINY, [1024], 1, 16, "int8", name="attend_1k_tiny"),
        # a decode step of sixteen sequences of up to 8 K
        _attend(LLAMA8B, _spread_lens(16, 8192, 1), 1, 16, "int8", name="attend_8k_16"),
        # a wide batch: 64 sequences of up to 4 K, blocks stored head-major
        _attend(QWEN14B, _spread_lens(64, 4096, 2), 1, 64, "e4m3", "head", name="attend_4k_64"),
        # a single very long, odd-sized context
        _attend(LLAMA8B, [131072 - 37], 1, 64, "int8", name="attend_128k_1"),
        # eight contexts of 8 K to 64 K tokens, three tokens of each at once (a draft being checked)
        _attend(LLAMA8B, RAGGED_CTX, 3, 32, "e4m3", name="attend_ragged8"),
        # a question of 57 tokens to a context of 16 K
        _attend(QWEN14B, [16384 + 57], 57, 16, "int8", name="attend_question"),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 2e14)


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "write", "read", "attend", "attend", "attend", "attend"])
    geometry = rng.choice([TINY, SMALL, LLAMA8B, LLAMA8B, QWEN14B, QWEN14B])
    D = geometry["head_dim"]
    block, type, layout = rng.choice([16, 16, 32, 64, 128]), rng.choice(["int8", "e4m3"]), rng.choice(["token", "head"])
    pairs, part = rng.choice(["half", "interleaved"]), rng.choice([D, D, D // 2, D // 4, 8 * rng.randint(1, D // 8)])
    scaling, norm = rng.choice(["none", "linear", "bands", "ramp"]), rng.random() < 0.5
    most = max(_cost(x) for x in listed())
    if kind == "rotate":
        return _rotate(geometry, spread(1, 8205), pairs, part, scaling, norm)
    if kind == "write":
        if rng.random() < 0.4:
            pairs, part, scaling, norm = "none", 0, "none", False
        return _write(geometry, spread(1, 16384), block, type, pairs, part, scaling, norm, layout)
    if kind == "read":
        if rng.random() < 0.25:
            pairs, part, scaling = "none", 0, "none"
        return _read(geometry, spread(1, 32768), block, type, pairs, part, scaling, layout)
    n = spread(1, 64)
    top = spread(1, 131072 if n == 1 else 65536)
    new = min(top, rng.choice([1, 1, 1, 2, 4, spread(1, 64)]))
    c = _attend(geometry, [rng.randint(max(new, top // 16), top) for _ in range(n)], new, block, type, layout)
    while _cost(c) > most or sum(_ints(c["lens"])) * geometry["kv_heads"] * D > 2 ** 28 or max(_ints(c["lens"])) * n > 2 ** 19:
        c["lens"] = _text([max(new, int(0.8 * t)) for t in _ints(c["lens"])])
        if max(_ints(c["lens"])) <= max(new, 64):
            break
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + salt)


def _normal(shape, seed, salt):
    return torch.randn(*shape, generator=_gen(seed, salt), device="cuda", dtype=torch.bfloat16)


def _i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _keys(rows, c, seed, salt):
    """[rows, H_kv, D]: unit normal keys around a drift of 64 tokens' length, as the keys of a text follow its topics."""
    Hkv, D = c["kv_heads"], c["head_dim"]
    drift = 0.7 * torch.randn((rows + 63) // 64, Hkv, D, generator=_gen(seed, salt + 1), device="cuda", dtype=torch.bfloat16)
    k = torch.randn(rows, Hkv, D, generator=_gen(seed, salt), device="cuda", dtype=torch.bfloat16) * 0.8
    return k + drift.repeat_interleave(64, 0)[:rows]


def _laid_out(x, layout):
    """[.., tokens, H_kv, D] in that order of memory, or as a view of head-major storage."""
    return x.transpose(-3, -2).contiguous().transpose(-3, -2) if layout == "head" else x.contiguous()


def _frequencies(part, scaling):
    """Angle per position of each pair, and what cosine and sine are multiplied by."""
    i = torch.arange(part // 2, dtype=torch.float64, device="cuda")
    theta, factor, length = 5.0e5, 8.0, 8192
    f = theta ** (-2 * i / max(part, 1))
    if scaling == "linear":                                  # all positions moved together
        return f / factor, 1.0
    if scaling == "bands":                                   # short waves as they are, long ones stretched, between them some of both
        keep = ((length * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 1.0
    if scaling == "ramp":                                    # likewise, by the pair's number, and a softmax that is as much sharper
        at = [part * math.log(length / (2 * math.pi * turns)) / (2 * math.log(theta)) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), part - 1)
        stretch = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f * (1 - stretch + stretch / factor), 0.1 * math.log(factor) + 1
    return f, 1.0


def _quantized(x, type):
    """8-bit values of [.., D] and the exponents [..] of their scales: the least from -100 on with which the type reaches all of them."""
    x = x.float()
    dtype, most = TYPES[type]
    f, t = math.frexp(most)
    m, e = torch.frexp(x.abs().amax(-1))                     # m 2^e <= f 2^t 2^exponent
    e = torch.where(m > 0, (e - t + (m > f)).clamp(min=-100), -100)
    y = torch.ldexp(x, -e[..., None])
    return (torch.round(y) if dtype is torch.int8 else y).to(dtype), e.to(torch.int8)


def _values(v, e):
    """What 8-bit values [.., D] and exponents [..] stand for."""
    return torch.ldexp(v.float(), e.int()[..., None])


def _store(c, n_blocks, seed, salt):
    """K, V [blocks, tokens, H_kv, D] in 8 bits and their exponents [blocks, H_kv, tokens]."""
    parts = []
    for n in range(2):
        x = (_keys if n == 0 else lambda rows, c, seed, salt: _normal((rows, c["kv_heads"], c["head_dim"]), seed, salt))(n_blocks * c["block"], c, seed, salt + 2 * n)
        values, exps = _quantized(x, c["type"])
        shape = (n_blocks, c["block"], c["kv_heads"])
        parts.append((_laid_out(values.view(*shape, c["head_dim"]).view(torch.int8), c["layout"]).view(TYPES[c["type"]][0]),
                      exps.view(shape).transpose(1, 2).contiguous()))
    return parts[0][0], parts[1][0], parts[0][1], parts[1][1]


def prepare(case, seed):
    c, kind = case, case["kind"]
    H, Hkv, D = c["heads"], c["kv_heads"], c["head_dim"]
    st = {"case": c}
    if own:
        from paper_2609_33503_b200 import binding as B
    if kind != "attend":
        n = c["rows"]
        st["pairs"] = c.get("pairs", "none")
        if st["pairs"] != "none":
            st["freq"], st["amplitude"] = _frequencies(c["part"], c["scaling"])
            span = 65536
            # (a chunk read back has moved as a whole, one way or the other)
            st["pos"] = (torch.randint(0, span, (n,), generator=_gen(seed, 4), device="cuda", dtype=torch.int32) if kind != "read" else
                         torch.randint(-span, span, ((n + 511) // 512,), generator=_gen(seed, 4), device="cuda", dtype=torch.int32)
                         .repeat_interleave(512)[:n].contiguous())
            if own:
                st["rotary"] = B.Rotary(st["freq"], interleaved=st["pairs"] == "interleaved", amplitude=st["amplitude"])
        st["wq"], st["wk"] = (1 + 0.1 * _normal((D,), seed, 30 + i) if c.get("norm") else None for i in range(2))
        st["eps"] = 1.0e-6
        if kind == "rotate" or (kind == "write" and st["pairs"] != "none"):
            st["q"] = _normal((n, H, D), seed, 20)
            st["q_out"] = torch.empty_like(st["q"])
        if kind == "rotate":
            st["k"] = _normal((n, Hkv, D), seed, 21)
            st["k_out"] = torch.empty_like(st["k"])
            return st
        # write, read: rows anywhere in a store that holds others, too
        n_blocks = -(-n // c["block"]) + 9
        st["store"] = _store(c, n_blocks, seed, 10)
        if kind == "write":
            st["k"], st["v"] = _laid_out(_keys(n, c, seed, 40), c["layout"]), _laid_out(_normal((n, Hkv, D), seed, 50), c["layout"])
            st["slots"] = torch.randperm(n_blocks * c["block"], generator=_gen(seed, 3), device="cuda")[:n].to(torch.int32)
        if kind == "read" or st["pairs"] == "none":          # whole blocks in any order
            blocks = torch.randperm(n_blocks, generator=_gen(seed, 5), device="cuda")[:, None] * c["block"]
            st["slots"] = (blocks + torch.arange(c["block"], device="cuda")).flatten()[:n].to(torch.int32)
        st["k_out"], st["v_out"] = (_laid_out(torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda"), c["layout"]) for _ in range(2))
        if own:
            st["paged"] = B.QuantizedStore(*st["store"])
        return st
    lens, new, bs = _ints(c["lens"]), c["new"], c["block"]
    have = [-(-t // bs) for t in lens]
    n_blocks = sum(have) + 5
    st["store"] = _store(c, n_blocks, seed, 60)
    perm = torch.randperm(n_blocks, generator=_gen(seed, 5), device="cuda").to(torch.int32)
    first = torch.tensor([0] + have, device="cuda").cumsum(0)[:-1]
    col = torch.arange(max(have), device="cuda")
    held = col[None] < torch.tensor(have, device="cuda")[:, None]
    st["table"] = torch.where(held, perm[(first[:, None] + col[None]).clamp(max=n_blocks - 1)], -1).to(torch.int32).contiguous()
    n = len(lens) * new
    st["row_cu"] = torch.arange(0, n + 1, new, dtype=torch.int32, device="cuda")
    st["row_seq"] = torch.arange(len(lens), dtype=torch.int32, device="cuda").repeat_interleave(new)
    st["row_len"] = (_i32(lens)[:, None] - new + 1 + torch.arange(new, dtype=torch.int32, device="cuda")).flatten().to(torch.int32).contiguous()
    st["max_len"] = max(lens)
    st["q"] = _normal((n, H, D), seed, 70)
    st["out"] = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(H, n, dtype=torch.float32, device="cuda")
    st["softmax_scale"] = D ** -0.5
    if own:
        st["paged"] = B.QuantizedStore(*st["store"])
        st["rows"] = B.ContinuationRows([0, len(lens)], [n], st["max_len"], st["row_cu"], st["row_seq"], st["row_len"], st["table"])
        nbytes = B.relaxkv_quantized_workspace_bytes(H, Hkv, D)
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
        off = (-ws.data_ptr()) % 256
        st["ws"] = ws[off:off + nbytes]
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------------

def _plain_turned(st, x, w=None):
    """Norm of the heads of [n, heads, D] and their rotation, in 32 bits."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * w.float()
    if st["pairs"] == "none":
        return x
    # (phases of tens of thousands of radians: reduced in 64 bits, as the tables that programs keep are)
    angle = st["pos"].double()[:, None] * st["freq"]
    cos, sin = ((f * st["amplitude"]).float()[:, None] for f in (angle.cos(), angle.sin()))
    part = 2 * st["freq"].shape[0]
    turned, rest = x[..., :part], x[..., part:]
    if st["pairs"] == "half":
        a, b = turned[..., :part // 2], turned[..., part // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = turned[..., 0::2], turned[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_rows(st, values, exps):
    """Rows of the store at the slots, as the values they stand for: [n, H_kv, D]."""
    bs = st["case"]["block"]
    block, at = st["slots"].long() // bs, st["slots"].long() % bs
    return _values(values.view(torch.int8)[block, at].view(values.dtype), exps[block, :, at])


def _plain_write(st):
    bs, type = st["case"]["block"], st["case"]["type"]
    block, at = st["slots"].long() // bs, st["slots"].long() % bs
    if "q" in st:
        st["q_out"].copy_(_plain_turned(st, st["q"], st["wq"]))
    for x, values, exps in ((_plain_turned(st, st["k"], st["wk"]), st["store"][0], st["store"][2]), (st["v"], st["store"][1], st["store"][3])):
        new, e = _quantized(x, type)
        values.view(torch.int8)[block, at] = new.view(torch.int8)
        exps[block, :, at] = e


def _plain_attend(st):
    """All sequences at once, padded to the longest: scores, masks, one softmax."""
    c = st["case"]
    H, Hkv, D = c["heads"], c["kv_heads"], c["head_dim"]
    n_seq = st["table"].shape[0]
    table = st["table"].clamp(min=0).long()
    k, v = (_values(x.view(torch.int8)[table].view(x.dtype), e[table].transpose(2, 3)) for x, e in (st["store"][0::2], st["store"][1::2]))
    k, v = k.flatten(1, 2), v.flatten(1, 2)                                                    # [sequences, tokens, H_kv, D]
    q = st["q"].float().view(n_seq, c["new"], Hkv, H // Hkv, D)
    s = torch.einsum("brkgd,btkd->bkrgt", q, k) * st["softmax_scale"]
    seen = torch.arange(k.shape[1], device="cuda") < st["row_len"].view(n_seq, c["new"], 1)
    s = s.masked_fill(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    o = torch.einsum("bkrgt,btkd->bkrgd", p, v) / z
    st["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(st["out"].shape))
    st["lse"].copy_((m + torch.log(z))[..., 0].permute(1, 3, 0, 2).reshape(st["lse"].shape))


# ---- one pass ---------------------------------------------------------------------------------------------------------------------

def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2609_33503_b200 import binding as B
    if kind == "rotate":
        if own:
            B.relaxkv_qk_norm_rotate(st["q"], st["k"], st["pos"], st["rotary"], st["q_out"], st["k_out"], st["wq"], st["wk"], st["eps"])
        else:
            st["q_out"].copy_(_plain_turned(st, st["q"], st["wq"]))
            st["k_out"].copy_(_plain_turned(st, st["k"], st["wk"]))
        return {"q": st["q_out"], "k": st["k_out"]}
    if kind == "write":
        if own:
            if "q" in st:
                B.relaxkv_append_quantized(st["paged"], st["k"], st["v"], st["slots"], q=st["q"], q_out=st["q_out"], positions=st["pos"],
                                           rotary=st["rotary"], w_q_norm=st["wq"], w_k_norm=st["wk"], eps=st["eps"])
            else:
                B.relaxkv_append_quantized(st["paged"], st["k"], st["v"], st["slots"])
            B.relaxkv_read_quantized(st["paged"], st["slots"], st["k_out"], st["v_out"])
        else:
            _plain_write(st)
            for out, values, exps in ((st["k_out"], st["store"][0], st["store"][2]), (st["v_out"], st["store"][1], st["store"][3])):
                out.copy_(_plain_rows(st, values, exps))
        out = {"k": st["k_out"], "v": st["v_out"]}
        return dict(out, q=st["q_out"]) if "q" in st else out
    if kind == "read":
        if own:
            B.relaxkv_read_quantized(st["paged"], st["slots"], st["k_out"], st["v_out"], positions=st.get("pos"), rotary=st.get("rotary"))
        else:
            st["k_out"].copy_(_plain_turned(st, _plain_rows(st, st["store"][0], st["store"][2])))
            st["v_out"].copy_(_plain_rows(st, st["store"][1], st["store"][3]))
        return {"k": st["k_out"], "v": st["v_out"]}
    if own:
        B.relaxkv_quantized_attention(st["paged"], st["rows"], st["q"], st["out"], st["ws"], lse_out=st["lse"], softmax_scale=st["softmax_scale"])
    else:
        _plain_attend(st)
    return {"out": st["out"], "lse": st["lse"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------------

def _exact_turned(st, x, w=None):
    """Pairs as complex numbers that are multiplied by amplitude * exp(i position frequency)."""
    x = x.double()
    if w is not None:
        x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + st["eps"])
    if st["pairs"] == "none":
        return x
    half = st["freq"].shape[0]
    turn = torch.polar(torch.full((1, 1), st["amplitude"], dtype=torch.float64, device="cuda"), st["pos"].double()[:, None] * st["freq"])[:, None]
    index = torch.arange(2 * half, device="cuda")
    first, second = (index[:half], index[half:]) if st["pairs"] == "half" else (index[0::2], index[1::2])
    y = torch.complex(x[..., first], x[..., second]) * turn
    x = x.clone()
    x[..., first], x[..., second] = y.real, y.imag
    return x


def _exact_values(x, type):
    """What [.., D] stands for when it is held in 8 bits: multiples of the scale, to the nearest one that the type has."""
    x = x.double()
    part, e = torch.frexp(x.abs().amax(-1, keepdim=True) / TYPES[type][1])                # (a logarithm may miss whole numbers)
    scale = torch.exp2(torch.where(part > 0, e - (part == 0.5).int(), -100).clamp(min=-100).double())
    y = x / scale
    if type == "int8":
        return torch.round(y) * scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)         # 3 bits behind the first; from 2^-6 down all alike
    return torch.round(y / step) * step * scale


def _exact_rows(st, at):
    out = []
    for values, exps in (st["store"][0::2], st["store"][1::2]):
        rows = values.float().double() * torch.exp2(exps.transpose(1, 2).double())[..., None]
        out.append(rows.flatten(0, 1)[at])
    return out


def _exact_attend(st):
    """Sequence by sequence and KV head by KV head, the tokens of a sequence put one behind the other."""
    c = st["case"]
    H, Hkv, D, new = c["heads"], c["kv_heads"], c["head_dim"], c["new"]
    G = H // Hkv
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for i, t in enumerate(_ints(c["lens"])):
        pages = st["table"][i, :-(-t // c["block"])].long()
        rows = slice(i * new, (i + 1) * new)
        hidden = torch.arange(t, device="cuda")[None] >= st["row_len"][rows, None]
        for g in range(Hkv):
            k, v = ((x.view(torch.int8)[pages, :, g].view(x.dtype).float().double() * torch.exp2(e[pages, g].double())[..., None]).reshape(-1, D)[:t]
                    for x, e in (st["store"][0::2], st["store"][1::2]))
            for h in range(g * G, (g + 1) * G):
                s = st["q"][rows, h].double() @ k.t() * st["softmax_scale"]
                s[hidden] = -math.inf
                lse[h, rows] = torch.logsumexp(s, -1)
                out[rows, h] = torch.softmax(s, -1) @ v
    return out, lse


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotate":
        return {"q": _exact_turned(st, st["q"], st["wq"]), "k": _exact_turned(st, st["k"], st["wk"])}
    if case["kind"] == "write":
        out = {"k": _exact_values(_exact_turned(st, st["k"], st["wk"]), case["type"]), "v": _exact_values(st["v"], case["type"])}
        return dict(out, q=_exact_turned(st, st["q"], st["wq"])) if "q" in st else out
    if case["kind"] == "read":
        k, v = _exact_rows(st, st["slots"].long())
        return {"k": _exact_turned(st, k), "v": v}
    out, lse = _exact_attend(st)
    return {"out": out, "lse": lse}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    H, Hkv, D = c["heads"], c["kv_heads"], c["head_dim"]
    token = Hkv * (2 * D + 2)                                # K, V and their exponents of one token in the store
    turns = 0 if c.get("pairs", "none") == "none" else 6
    if kind == "rotate":                                     # Q and K in and out, a position per row
        return {"bytes": c["rows"] * (2 * 2 * (H + Hkv) * D + 4), "flops": c["rows"] * (H + Hkv) * D * (3 + (4 if c["norm"] else 0))}
    if kind == "write":                                      # K and V in, into the store and back in bf16; Q in and out
        q = 4 * H * D + 4 if turns else 0
        return {"bytes": c["rows"] * (2 * 2 * 2 * Hkv * D + token + q + 4), "flops": c["rows"] * ((H if turns else 0) + 2 * Hkv) * D * 4}
    if kind == "read":
        return {"bytes": c["rows"] * (token + 2 * 2 * Hkv * D + 4 + (4 if turns else 0)), "flops": c["rows"] * 2 * Hkv * D * 4}
    lens, new = _ints(c["lens"]), c["new"]
    pairs = sum((t - new + 1 + j) for t in lens for j in range(new))
    n = len(lens) * new
    return {"bytes": sum(lens) * token + n * (4 * H * D + 4 * H) + 4 * sum(-(-t // c["block"]) for t in lens), "flops": 4 * H * D * pairs}
