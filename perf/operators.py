"""Operators for many continuations of a repaired context, as measurable cases.

A repaired context is paid for once and answered from many times: several samples, beams or follow-up questions continue it.
The context stays in its contiguous cache; what each continuation adds of its own lives in a paged store.  Five kinds of pass:

  tables   block tables and slot maps of a step from the sequences' lengths (`relaxkv_build_block_tables`)
  append   norm of the query and key heads, rotation, append of K and V to the paged store (`relaxkv_qk_norm_rope_append_paged`)
  prefix   attention of all rows over the shared context, read once for all, and over their own paged tokens
           (`relaxkv_shared_prefix_attention`)
  bounds   8-bit bounds of the keys of every context block (`relaxkv_block_bounds`)
  sparse   blocks of the highest bound for each row and KV head, and attention over those and the row's own tokens
           (`relaxkv_select_blocks`, `relaxkv_block_sparse_attention`)

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


def _text(xs):
    return ",".join(str(int(x)) for x in xs)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _tables(n_seq, stored, new, block, **kw):
    """stored, new: the longest own length and the most new tokens of a sequence."""
    return dict(kind="tables", n_seq=n_seq, stored=stored, new=new, block=block, **kw)


def _append(geometry, rows, block, norm, layout="token", **kw):
    return dict(kind="append", rows=rows, block=block, norm=norm, layout=layout, **geometry, **kw)


def _attend(kind, geometry, ctx, seqs, stored, block, *, new=1, ctx_layout="token", layout="token", ctx_block=64, select=0, **kw):
    """ctx: tokens of each context; seqs: continuations of each; stored: the longest own length; new: rows of each sequence."""
    c = dict(kind=kind, ctx=_text(ctx), seqs=_text(seqs), stored=stored, block=block, new=new, ctx_layout=ctx_layout, layout=layout,
             **geometry, **kw)
    return dict(c, ctx_block=ctx_block, select=select) if kind == "sparse" else c


def _bounds(geometry, ctx, ctx_block, ctx_layout="token", **kw):
    return dict(kind="bounds", ctx=_text(ctx), ctx_block=ctx_block, ctx_layout=ctx_layout, **geometry, **kw)


def listed():
    return [
        # a decode step of 64 running sequences: one token each, a new block now and then; launch latency
        _tables(64, 900, 1, 16, name="tables_decode"),
        # 2000 sequences brought in at once, up to 500 tokens each, some of them ending
        _tables(2000, 3000, 500, 16, name="tables_prompts"),
        # one decode step's rows of one layer
        _append(LLAMA8B, 64, 16, False, name="append_decode"),
        # the rows of a long prompt chunk, with the head norms of the larger model, head-major blocks
        _append(QWEN14B, 8205, 64, True, "head", name="append_chunk"),
        # the smallest call: four samples of a 1K context
        _attend("prefix", TINY, [1024], [4], 20, 16, name="prefix_1k_tiny"),
        # sixteen samples of one 16K context, own answers up to 300 tokens
        _attend("prefix", LLAMA8B, [16384], [16], 300, 16, name="prefix_16k_16"),
        # a wide batch: 64 samples of a 32K context, answers up to 1K tokens, both stored head-major
        _attend("prefix", QWEN14B, [32768], [64], 1024, 64, ctx_layout="head", layout="head", name="prefix_32k_64"),
        # eight contexts of 8K to 64K tokens, one to 24 continuations each, two tokens of each at once (a draft being checked)
        _attend("prefix", LLAMA8B, RAGGED_CTX, (1, 24, 3, 8, 16, 2, 5, 4), 400, 32, new=2, name="prefix_ragged8"),
        # bounds of one repaired 16K layer, and of one very long, odd-sized context
        _bounds(LLAMA8B, [16384], 64, name="bounds_16k"),
        _bounds(QWEN14B, [131072 - 37], 32, "head", name="bounds_128k"),
        # few samples of a 32K context, an eighth of its blocks each
        _attend("sparse", QWEN14B, [32768], [4], 300, 16, ctx_block=64, select=64, name="sparse_32k_4"),
        # two very long contexts with eight samples each, one sixteenth of the blocks
        _attend("sparse", LLAMA8B, [131072 - 37, 100000], [8, 8], 600, 32, ctx_layout="head", ctx_block=64, select=128, name="sparse_128k_16"),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 8e14)


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["tables", "append", "prefix", "prefix", "prefix", "bounds", "sparse", "sparse"])
    geometry = rng.choice([TINY, SMALL, LLAMA8B, LLAMA8B, QWEN14B, QWEN14B])
    block = rng.choice([16, 16, 32, 64, 128])
    layout, ctx_layout = rng.choice(["token", "head"]), rng.choice(["token", "head"])
    most = max(_cost(x) for x in listed())
    if kind == "tables":
        return _tables(spread(1, 4096), spread(1, 4000), spread(1, 250), block)
    if kind == "append":
        return _append(geometry, spread(1, 8205), block, rng.random() < 0.5, layout)
    n_ctx = 1 if rng.random() < 0.5 else rng.randint(2, 8)
    ctx = [spread(256, 131072 if n_ctx == 1 else 65536) for _ in range(n_ctx)]
    if kind == "bounds":
        c = _bounds(geometry, ctx, rng.choice([16, 32, 64, 64, 128]), ctx_layout)
    else:
        seqs = [spread(1, 64 if n_ctx == 1 else 16) for _ in range(n_ctx)]
        c = _attend(kind, geometry, ctx, seqs, spread(1, 1024), block, new=rng.choice([1, 1, 1, 2, 4]), ctx_layout=ctx_layout, layout=layout,
                    ctx_block=rng.choice([16, 32, 64, 64, 128]), select=spread(4, 128))
    while _cost(c) > most:
        ctx = [max(256, int(0.8 * t)) for t in ctx]
        c["ctx"] = _text(ctx)
        if kind != "bounds":
            c["seqs"] = _text([max(1, int(0.9 * s)) for s in _ints(c["seqs"])])
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
    drift = 0.7 * torch.randn((rows + 63) // 64, Hkv, D, generator=_gen(seed, salt + 1), device="cuda")
    k = torch.randn(rows, Hkv, D, generator=_gen(seed, salt), device="cuda") * 0.8
    return (k + drift.repeat_interleave(64, 0)[:rows]).to(torch.bfloat16)


def _laid_out(x, layout):
    """[.., tokens, H_kv, D] in that order of memory, or as a view of head-major storage."""
    return x.transpose(-3, -2).contiguous().transpose(-3, -2) if layout == "head" else x.contiguous()


def _lengths(c):
    """(stored, new) tokens of every sequence: which ones does not depend on the seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    if c["kind"] == "tables":
        stored = [rng.randint(0, c["stored"]) for _ in range(c["n_seq"])]
        new = [rng.randint(1, c["new"]) for _ in stored]
        if c["new"] > 1:                       # a batch in motion: some sequences end, some wait
            new = [-1 if rng.random() < 0.1 else 0 if rng.random() < 0.1 else n for n in new]
        return stored, new
    n = sum(_ints(c["seqs"]))
    return [rng.randint(0, c["stored"]) for _ in range(n)], [c["new"]] * n


def _store(c, n_blocks, seed, salt):
    shape = (n_blocks, c["block"], c["kv_heads"], c["head_dim"])
    return [_laid_out(_normal(shape, seed, salt + n), c["layout"]) for n in range(2)]


def prepare(case, seed):
    c, kind = case, case["kind"]
    st = {"case": c}
    if kind == "tables":
        stored, new = _lengths(c)
        bs = c["block"]
        have = [-(-s // bs) for s in stored]
        need = [-(-(s + n) // bs) - h if n > 0 else 0 for s, n, h in zip(stored, new, have)]
        total = sum(have) + sum(need) + 7
        perm = torch.randperm(total, generator=_gen(seed, 1), device="cuda").to(torch.int32)
        width = max(h + m for h, m in zip(have, need)) + 1
        table = torch.full((c["n_seq"], width), -1, dtype=torch.int32, device="cuda")
        first = torch.tensor([0] + have, device="cuda").cumsum(0)
        col = torch.arange(width, device="cuda")
        held = col[None] < torch.tensor(have, device="cuda")[:, None]
        table[held] = perm[(first[:-1, None] + col[None])[held]]
        n_free = total - sum(have)
        free = torch.full((total,), -1, dtype=torch.int32, device="cuda")
        free[:n_free] = perm[sum(have):]
        base = torch.randint(0, 65536, (c["n_seq"],), generator=_gen(seed, 2), device="cuda", dtype=torch.int32)
        n_rows = sum(n for n in new if n > 0)
        e = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
        st.update(seq_len=_i32(stored), new_len=_i32(new), seq_base=base, free=free, n_free=_i32([n_free]), table=table,
                  out=dict(row_cu=e(c["n_seq"] + 1), row_seq=e(n_rows), row_pos=e(n_rows), row_len=e(n_rows), row_slot=e(n_rows),
                           seq_len=e(c["n_seq"]), n_free=e(1)))
        return st
    H, Hkv, D = c["heads"], c["kv_heads"], c["head_dim"]
    if kind == "append":
        n, bs = c["rows"], c["block"]
        n_blocks = -(-n // bs) + 9
        st["store"] = _store(c, n_blocks, seed, 10)
        st["q"], st["k"], st["v"] = (_normal((n, h, D), seed, 20 + i) for i, h in enumerate((H, Hkv, Hkv)))
        st["slots"] = torch.randperm(n_blocks * bs, generator=_gen(seed, 3), device="cuda")[:n].to(torch.int32)
        st["pos"] = torch.randint(0, 65536, (n,), generator=_gen(seed, 4), device="cuda", dtype=torch.int32)
        st["wq"], st["wk"] = (1 + 0.1 * _normal((D,), seed, 30 + i) if c["norm"] else None for i in range(2))
        st["theta"], st["eps"] = 1.0e6, 1.0e-6
        st["q_out"] = torch.empty_like(st["q"])
        if own:
            from paper_2609_33503_b200 import binding as B
            st["paged"] = B.PagedStore(*st["store"])
        return st
    ctx = _ints(c["ctx"])
    st["ctx_at"] = [sum(ctx[:b]) for b in range(len(ctx))]
    st["k"] = _laid_out(_keys(sum(ctx), c, seed, 40), c["ctx_layout"])
    if kind == "bounds":
        nb = sum(-(-t // c["ctx_block"]) for t in ctx)
        st["bounds"] = torch.empty(nb, Hkv, 2, D, dtype=torch.int8, device="cuda")
        st["scale"] = torch.empty(nb, Hkv, dtype=torch.float32, device="cuda")
        if own:
            from paper_2609_33503_b200 import binding as B
            st["shape"], st["view"] = B.Shape(H, Hkv, D, ctx), B.CacheView(st["k"], None, st["ctx_at"])
        return st
    # prefix / sparse: contexts, the paged store with the sequences' own tokens in shuffled blocks, one or a few rows of each
    st["v"] = _laid_out(_normal((sum(ctx), Hkv, D), seed, 50), c["ctx_layout"])
    seqs, bs = _ints(c["seqs"]), c["block"]
    stored, new = _lengths(c)
    have = [-(-(s + n) // bs) for s, n in zip(stored, new)]
    n_blocks = sum(have) + 5
    st["store"] = _store(c, n_blocks, seed, 60)
    perm = torch.randperm(n_blocks, generator=_gen(seed, 5), device="cuda").to(torch.int32)
    width = max(have)
    table = torch.full((len(have), width), -1, dtype=torch.int32)
    for i, h in enumerate(have):
        table[i, :h] = torch.arange(sum(have[:i]), sum(have[:i]) + h)
    table = table.cuda()
    st["table"] = torch.where(table >= 0, perm[table.clamp(min=0).long()], table).contiguous()
    st["seq_cu"] = [sum(seqs[:b]) for b in range(len(seqs) + 1)]
    row_seq = [i for i, n in enumerate(new) for _ in range(n)]
    row_len = [stored[i] + j + 1 for i, n in enumerate(new) for j in range(n)]
    st["row_cu"] = _i32([sum(new[:i]) for i in range(len(new) + 1)])
    st["row_seq"], st["row_len"] = _i32(row_seq), _i32(row_len)
    st["max_rows"] = [s * c["new"] for s in seqs]
    st["max_len"] = max(row_len)
    n = len(row_seq)
    st["q"] = _normal((n, H, D), seed, 70)
    st["out"] = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(H, n, dtype=torch.float32, device="cuda")
    st["softmax_scale"] = D ** -0.5
    if kind == "sparse":
        st["bounds"], st["scale"] = _plain_bounds(st["k"], ctx, c["ctx_block"])
        st["first"], st["last"] = 1, min(2, c["select"] - 1)
        st["blocks"] = torch.empty(n, Hkv, c["select"], dtype=torch.int32, device="cuda")
    if own:
        from paper_2609_33503_b200 import binding as B
        st["shape"], st["view"] = B.Shape(H, Hkv, D, ctx), B.CacheView(st["k"], st["v"], st["ctx_at"])
        st["paged"] = B.PagedStore(*st["store"])
        st["rows"] = B.ContinuationRows(st["seq_cu"], st["max_rows"], st["max_len"], st["row_cu"], st["row_seq"], st["row_len"], st["table"])
        nbytes = B.relaxkv_continuation_workspace_bytes(st["shape"], n, c.get("ctx_block", 0))
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
        off = (-ws.data_ptr()) % 256
        st["ws"] = ws[off:off + nbytes]
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------------

def _plain_tables(st):
    bs, table, o = st["case"]["block"], st["table"], st["out"]
    length, new, free, n_free = st["seq_len"].long(), st["new_len"].long(), st["free"], st["n_free"].long()
    have = (length + bs - 1) // bs
    ends, grow = new < 0, new.clamp(min=0)
    need = torch.where(ends, 0, (length + grow + bs - 1) // bs - have)
    back = torch.where(ends, have, 0)
    col = torch.arange(table.shape[1], device="cuda")
    at = torch.arange(free.shape[0], device="cuda")
    held = (col[None] < back[:, None])
    stack = free.clone()                                                    # released blocks go on top of the free ones
    top = n_free + held.sum()
    stack[(at >= n_free) & (at < top)] = table[held]
    fresh = (col[None] >= have[:, None]) & (col[None] < (have + need)[:, None])
    table[fresh] = stack[top - 1 - torch.arange(int(fresh.sum()), device="cuda")]
    left = top - need.sum()
    free[(at >= n_free) & (at < left)] = stack[(at >= n_free) & (at < left)]
    row_cu = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), grow.cumsum(0)])
    seq = torch.repeat_interleave(torch.arange(len(grow), device="cuda"), grow)
    index = length[seq] + torch.arange(len(seq), device="cuda") - row_cu[seq]
    values = dict(row_cu=row_cu, row_seq=seq, row_pos=st["seq_base"].long()[seq] + index, row_len=index + 1,
                  row_slot=table[seq, index // bs].long() * bs + index % bs, seq_len=torch.where(ends, 0, length + grow), n_free=left)
    for name, v in values.items():
        o[name].copy_(v)


def _plain_append(st):
    def rotated(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * w.float()
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)

    half = st["case"]["head_dim"] // 2
    # (phases of tens of thousands of radians: reduced in 64 bits, as the tables that programs keep are)
    angle = st["pos"].double()[:, None] * st["theta"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    st["q_out"].copy_(rotated(st["q"], st["wq"]))
    bs = st["case"]["block"]
    block, at = st["slots"].long() // bs, st["slots"].long() % bs
    st["store"][0][block, at] = rotated(st["k"], st["wk"])
    st["store"][1][block, at] = st["v"]


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 127 s; 1 where amax is 0."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 127 / 128, e - 7, e - 6).clamp(min=-100)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), 1.0)


def _plain_bounds(k, ctx, bs):
    his, los, at = [], [], 0
    for t in ctx:
        x = k[at:at + t].float()
        at += t
        nb, Hkv, D = -(-t // bs), x.shape[1], x.shape[2]
        for out, fill, reduce in ((his, -math.inf, torch.amax), (los, math.inf, torch.amin)):
            full = torch.full((nb * bs, Hkv, D), fill, device="cuda")
            full[:t] = x
            out.append(reduce(full.view(nb, bs, Hkv, D), 1))
    hi, lo = torch.cat(his), torch.cat(los)
    scale = _pow2_scale(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    bounds = torch.stack([torch.ceil(hi / scale[..., None]), torch.floor(lo / scale[..., None])], 2)
    return bounds.to(torch.int8), scale


def _plain_select(st):
    c = st["case"]
    R, H, D = st["q"].shape
    Hkv, n_sel, bs = c["kv_heads"], c["select"], c["ctx_block"]
    q = st["q"].float().view(R, Hkv, H // Hkv, D)
    sq = _pow2_scale(q.abs().amax(-1))
    qi = torch.round(q / sq[..., None])
    row, at, lists = 0, 0, []
    for t, n in zip(_ints(c["ctx"]), st["max_rows"]):
        nb = -(-t // bs)
        hi, lo = st["bounds"][at:at + nb, :, 0].float(), st["bounds"][at:at + nb, :, 1].float()
        x = qi[row:row + n]
        dot = torch.einsum("rkgd,bkd->rkgb", x.clamp(min=0), hi) + torch.einsum("rkgd,bkd->rkgb", x.clamp(max=0), lo)
        score = (dot * sq[row:row + n, ..., None]).amax(2) * st["scale"][at:at + nb].t()[None]
        score[..., :st["first"]] = math.inf
        score[..., max(0, nb - st["last"]):] = math.inf
        best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :n_sel].sort(-1)[0]
        lists.append(torch.nn.functional.pad(best, (0, n_sel - best.shape[-1]), value=-1))
        row, at = row + n, at + nb
    st["blocks"].copy_(torch.cat(lists))


def _plain_attention(st, blocks=None):
    """Rows of one context at a time: scores over the context (or its listed blocks) and over the rows' own tokens, one softmax."""
    c = st["case"]
    H, Hkv, D, bs, scale = c["heads"], c["kv_heads"], c["head_dim"], c["block"], st["softmax_scale"]
    G, row = H // Hkv, 0
    for b, (t, n) in enumerate(zip(_ints(c["ctx"]), st["max_rows"])):
        at, rows = st["ctx_at"][b], slice(row, row + n)
        k, v = st["k"][at:at + t], st["v"][at:at + t]
        q = st["q"][rows].float().view(n, Hkv, G, D)
        if blocks is None:
            s_ctx = torch.einsum("rkgd,tkd->rkgt", q, k.float()) * scale
        else:
            cb = c["ctx_block"]
            token = (blocks[rows].long()[..., None] * cb + torch.arange(cb, device="cuda")).flatten(2)        # [n, Hkv, select * cb]
            valid = (token >= 0) & (token < t)
            index = token.clamp(0, t - 1)
            head = torch.arange(Hkv, device="cuda")[None, :, None]
            s_ctx = torch.einsum("rkgd,rktd->rkgt", q, k[index, head].float()) * scale
            s_ctx = s_ctx.masked_fill(~valid[:, :, None], -math.inf)
        table = st["table"][st["row_seq"][rows].long()].clamp(min=0).long()
        own_k, own_v = (x[table].flatten(1, 2).float() for x in st["store"])                                  # [n, width * bs, Hkv, D]
        s_own = torch.einsum("rkgd,rtkd->rkgt", q, own_k) * scale
        seen = torch.arange(own_k.shape[1], device="cuda")[None] < st["row_len"][rows, None]
        s_own = s_own.masked_fill(~seen[:, None, None], -math.inf)
        m = torch.maximum(s_ctx.amax(-1, keepdim=True), s_own.amax(-1, keepdim=True))
        p_ctx, p_own = torch.exp(s_ctx - m), torch.exp(s_own - m)
        z = p_ctx.sum(-1, keepdim=True) + p_own.sum(-1, keepdim=True)
        if blocks is None:
            o = torch.einsum("rkgt,tkd->rkgd", p_ctx, v.float())
        else:
            o = torch.einsum("rkgt,rktd->rkgd", p_ctx, v[index, head].float())
        o = (o + torch.einsum("rkgt,rtkd->rkgd", p_own, own_v)) / z
        st["out"][rows].copy_(o.reshape(n, H, D))
        st["lse"][:, rows].copy_((m + torch.log(z)).reshape(n, H).t())
        row += n


# ---- one pass ---------------------------------------------------------------------------------------------------------------------

def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2609_33503_b200 import binding as B
    if kind == "tables":
        o = st["out"]
        if own:
            B.relaxkv_build_block_tables(st["case"]["block"], st["seq_len"], st["new_len"], st["seq_base"], st["free"], st["n_free"], st["table"],
                                         o["seq_len"], o["n_free"], o["row_cu"], o["row_seq"], o["row_pos"], o["row_len"], o["row_slot"])
        else:
            _plain_tables(st)
        return dict(o, table=st["table"], free=st["free"])
    if kind == "append":
        if own:
            B.relaxkv_qk_norm_rope_append_paged(st["paged"], st["q"], st["k"], st["v"], st["pos"], st["slots"], st["theta"], st["q_out"],
                                                st["wq"], st["wk"], st["eps"])
        else:
            _plain_append(st)
        return {"q": st["q_out"], "k": st["store"][0], "v": st["store"][1]}
    if kind == "bounds":
        if own:
            B.relaxkv_block_bounds(st["shape"], st["view"], st["case"]["ctx_block"], st["bounds"], st["scale"])
            bounds, scale = st["bounds"], st["scale"]
        else:
            bounds, scale = _plain_bounds(st["k"], _ints(st["case"]["ctx"]), st["case"]["ctx_block"])
        return {"bounds": bounds * scale[..., None, None], "scale": scale}
    if kind == "sparse":
        if own:
            B.relaxkv_select_blocks(st["shape"], st["case"]["ctx_block"], st["bounds"], st["scale"], st["rows"], st["q"], st["first"], st["last"],
                                    st["blocks"], st["ws"])
            B.relaxkv_block_sparse_attention(st["shape"], st["view"], st["paged"], st["rows"], st["case"]["ctx_block"], st["blocks"], st["q"],
                                             st["out"], st["ws"], lse_out=st["lse"])
        else:
            _plain_select(st)
            _plain_attention(st, st["blocks"])
        return {"out": st["out"], "lse": st["lse"], "blocks": st["blocks"]}
    if own:
        B.relaxkv_shared_prefix_attention(st["shape"], st["view"], st["paged"], st["rows"], st["q"], st["out"], st["ws"], lse_out=st["lse"])
    else:
        _plain_attention(st)
    return {"out": st["out"], "lse": st["lse"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------------

def _exact_scale(amax):
    """2^ceil(log2(amax / 127)), from -100 on; 1 for 0."""
    e = torch.log2(amax / 127).ceil().clamp(min=-100)
    return torch.where(amax > 0, torch.exp2(e), 1.0).double()


def _exact_bounds(k, ctx, bs):
    values, scales, at = [], [], 0
    for t in ctx:
        for first in range(0, t, 512 * bs):                                  # whole blocks, then the short one by itself
            part = k[at + first:at + min(t, first + 512 * bs)].double()
            whole = part.shape[0] // bs * bs
            for x in ([part[:whole].unflatten(0, (-1, bs))] if whole else []) + ([part[None, whole:]] if whole < part.shape[0] else []):
                hi, lo = x.max(1)[0], x.min(1)[0]
                s = _exact_scale(torch.maximum(hi.abs().max(-1)[0], lo.abs().max(-1)[0]))[..., None]
                values.append(torch.stack([torch.ceil(hi / s) * s, torch.floor(lo / s) * s], -2))
                scales.append(s[..., 0])
        at += t
    return torch.cat(values), torch.cat(scales)


def _exact_select(st):
    """Every (row, KV head) by itself: blocks ordered by (score falling, index rising)."""
    c = st["case"]
    H, Hkv, bs = c["heads"], c["kv_heads"], c["ctx_block"]
    G, row, at, out = H // Hkv, 0, 0, torch.full_like(st["blocks"], -1)
    for t, n in zip(_ints(c["ctx"]), st["max_rows"]):
        nb = -(-t // bs)
        bound = st["bounds"][at:at + nb].double() * st["scale"][at:at + nb, :, None, None].double()
        for r in range(row, row + n):
            for g in range(Hkv):
                q = st["q"][r, g * G:(g + 1) * G].double()
                s = _exact_scale(q.abs().max(-1)[0])[:, None]
                q = torch.round(q / s) * s
                best = torch.maximum(q[:, None] * bound[None, :, g, 0], q[:, None] * bound[None, :, g, 1]).sum(-1).max(0)[0]
                best[:st["first"]] = math.inf
                best[max(0, nb - st["last"]):] = math.inf
                order = torch.argsort(-best, stable=True)[:c["select"]]
                out[r, g, :len(order)] = order.sort()[0].to(torch.int32)
        row, at = row + n, at + nb
    return out


def _exact_attention(st, blocks=None):
    """Row by row and KV head by KV head, with the keys of a row put one behind the other."""
    c = st["case"]
    H, Hkv, D, bs = c["heads"], c["kv_heads"], c["head_dim"], c["block"]
    G, n_rows = H // Hkv, st["q"].shape[0]
    out = torch.empty(n_rows, H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(H, n_rows, dtype=torch.float64, device="cuda")
    row_seq, row_len, row = st["row_seq"].tolist(), st["row_len"].tolist(), 0
    for b, (t, n) in enumerate(zip(_ints(c["ctx"]), st["max_rows"])):
        at = st["ctx_at"][b]
        for g in range(Hkv):
            k_ctx, v_ctx = (st[x][at:at + t, g].double() for x in "kv")
            for r in range(row, row + n):
                pages = st["table"][row_seq[r], :-(-row_len[r] // bs)].long()
                k_own, v_own = (x[pages, :, g].reshape(-1, D)[:row_len[r]].double() for x in st["store"])
                if blocks is None:
                    k, v = torch.cat([k_ctx, k_own]), torch.cat([v_ctx, v_own])
                else:
                    x = blocks[r, g].long()
                    token = (x[x >= 0, None] * c["ctx_block"] + torch.arange(c["ctx_block"], device="cuda")).flatten()
                    token = token[token < t]
                    k, v = torch.cat([k_ctx[token], k_own]), torch.cat([v_ctx[token], v_own])
                s = st["q"][r, g * G:(g + 1) * G].double() @ k.t() * st["softmax_scale"]
                lse[g * G:(g + 1) * G, r] = torch.logsumexp(s, -1)
                out[r, g * G:(g + 1) * G] = torch.softmax(s, -1) @ v
        row += n
    return out, lse


def _exact_append(st):
    c = st["case"]
    half = c["head_dim"] // 2
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                       st["pos"].double()[:, None] * torch.exp(-math.log(st["theta"]) * torch.arange(half, device="cuda").double() / half))

    def rotated(x, w):
        x = x.double()
        if w is not None:
            x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + st["eps"])
        y = torch.complex(x[..., :half], x[..., half:]) * turn[:, None]
        return torch.cat([y.real, y.imag], -1)

    k, v = (x.double() for x in st["store"])
    for i, slot in enumerate(st["slots"].tolist()):
        if i == 0:
            new_k = rotated(st["k"], st["wk"])
        k[slot // c["block"], slot % c["block"]] = new_k[i]
        v[slot // c["block"], slot % c["block"]] = st["v"][i].double()
    return {"q": rotated(st["q"], st["wq"]), "k": k, "v": v}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "tables":                            # whole numbers: equal or wrong
        return None
    if case["kind"] == "append":
        return _exact_append(st)
    if case["kind"] == "bounds":
        bounds, scale = _exact_bounds(st["k"], _ints(case["ctx"]), case["ctx_block"])
        return {"bounds": bounds, "scale": scale}
    blocks = _exact_select(st) if case["kind"] == "sparse" else None
    out, lse = _exact_attention(st, blocks)
    return {"out": out, "lse": lse} if blocks is None else {"out": out, "lse": lse, "blocks": blocks}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    if kind == "tables":
        stored, new = _lengths(c)
        bs = c["block"]
        rows = sum(n for n in new if n > 0)
        moved = sum(-(-(s + n) // bs) - -(-s // bs) if n > 0 else -(-s // bs) if n < 0 else 0 for s, n in zip(stored, new))
        return {"bytes": 4 * (5 * c["n_seq"] + 2 * moved + 4 * rows), "flops": 0}
    H, Hkv, D = c["heads"], c["kv_heads"], c["head_dim"]
    if kind == "append":                                    # Q, K, V in; Q, K, V out; position and slot of every row
        return {"bytes": c["rows"] * (2 * 2 * (H + 2 * Hkv) * D + 8), "flops": c["rows"] * (H + Hkv) * D * 8}
    ctx = _ints(c["ctx"])
    if kind == "bounds":
        blocks = sum(-(-t // c["ctx_block"]) for t in ctx)
        return {"bytes": sum(ctx) * Hkv * D * 2 + blocks * Hkv * (2 * D + 4), "flops": 2 * sum(ctx) * Hkv * D}
    stored, new = _lengths(c)
    seqs, kv = _ints(c["seqs"]), 4 * Hkv * D
    n_rows = sum(new)
    own_bytes = sum(s + n for s, n in zip(stored, new)) * kv + n_rows * (4 * H * D + 4 * H)
    own_keys = sum(s + j + 1 for s, n in zip(stored, new) for j in range(n))
    if kind == "prefix":
        return {"bytes": sum(ctx) * kv + own_bytes, "flops": 4 * H * D * (sum(t * s * c["new"] for t, s in zip(ctx, seqs)) + own_keys)}
    listed_keys = sum(s * c["new"] * min(t, c["select"] * c["ctx_block"]) for t, s in zip(ctx, seqs))
    blocks = [-(-t // c["ctx_block"]) for t in ctx]
    # rows of one context may list the same blocks: at the most, the context is read once
    read = sum(min(t, s * c["new"] * c["select"] * c["ctx_block"]) for t, s in zip(ctx, seqs))
    return {"bytes": read * kv + own_bytes + sum(blocks) * Hkv * (2 * D + 4) + 4 * n_rows * Hkv * c["select"],
            "flops": 4 * H * D * (listed_keys + own_keys) + 4 * H * D * sum(x * s * c["new"] for x, s in zip(blocks, seqs))}
