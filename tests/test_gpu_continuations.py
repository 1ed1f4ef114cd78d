"""Operators over continuations on the GPU against their plain 64-bit forms (tests/continuation_oracle.py)."""
import numpy as np
import pytest
import torch

from tests import continuation_oracle as orc

pytestmark = pytest.mark.gpu


def B():
    from paper_2609_33503_b200 import binding
    return binding


def status():
    torch.cuda.synchronize()
    return B().relaxkv_read_device_status()[0]


def i32(xs):
    return torch.tensor(np.asarray(xs).tolist(), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def workspace(nbytes):
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
    off = (-ws.data_ptr()) % 256
    return ws[off:off + nbytes]


# ---- block tables ---------------------------------------------------------------------------------------------------------------

def build(bs, seq_len, new_len, base, free, n_free, table, n_rows):
    e = lambda n, v=-9: torch.full((max(n, 0),), v, dtype=torch.int32, device="cuda")
    n = len(seq_len)
    t, fr = i32(table), i32(free) if len(free) else e(0)
    o = dict(seq_len=e(n), n_free=e(1), row_cu=e(n + 1), row_seq=e(n_rows), row_pos=e(n_rows), row_len=e(n_rows), row_slot=e(n_rows))
    B().relaxkv_build_block_tables(bs, i32(seq_len), i32(new_len), None if base is None else i32(base), fr, i32([n_free]), t, o["seq_len"], o["n_free"],
                                   o["row_cu"], o["row_seq"], o["row_pos"], o["row_len"], o["row_slot"])
    return dict({k: v.cpu().tolist() for k, v in o.items()}, table=t.cpu().tolist(), free=fr.cpu().tolist())


def check_build(bs, seq_len, new_len, base, free, n_free, table, n_rows, got):
    cu, rows, lens, left, stack, tab = orc.block_tables(bs, seq_len, new_len, [0] * len(seq_len) if base is None else base, free, n_free, table, n_rows)
    assert got["row_cu"] == cu and got["seq_len"] == lens and got["n_free"] == [left] and got["free"] == stack and got["table"] == tab
    pad = [(-1, 0, 0, -1)] * (n_rows - len(rows))
    assert list(zip(got["row_seq"], got["row_pos"], got["row_len"], got["row_slot"])) == rows + pad


def random_state(rng, n, bs, longest, width=None):
    lens = [int(x) for x in rng.integers(0, longest + 1, n)]
    have = [-(-x // bs) for x in lens]
    width = width or max(have) + 40
    ids = rng.permutation(sum(have) + 60 * n + 5).tolist()
    table = [[ids.pop() for _ in range(h)] + [-1] * (width - h) for h in have]
    return lens, table, ids


@pytest.mark.parametrize("n,bs,longest,most,seed", [(1, 16, 0, 1, 0), (1, 16, 100, 1, 1), (5, 128, 300, 3, 2), (64, 16, 900, 1, 3), (33, 32, 77, 90, 4),
                                                    (777, 16, 200, 40, 5), (4096, 64, 500, 9, 6),
                                                    (120, 128, 100, 1000, 7), (256, 32, 60, 2, 8), (257, 32, 60, 2, 9), (1025, 16, 40, 3, 10)])
def test_block_tables(n, bs, longest, most, seed):
    rng = np.random.default_rng(seed)
    lens, table, free = random_state(rng, n, bs, longest)
    new = [int(x) for x in rng.integers(0, most + 1, n)]
    if n > 3:
        for i in rng.choice(n, n // 4, replace=False):
            new[i] = -1
    base = [int(x) for x in rng.integers(0, 100000, n)]
    rows = sum(x for x in new if x > 0)
    cap = free + [-5] * (sum(-(-x // bs) for x in lens))
    args = (bs, lens, new, base, cap, len(free), table, rows + (3 if seed % 2 else 0))
    check_build(*args, build(*args))
    assert status() == B().OK


def test_block_tables_take_ended_blocks_again_and_fill_the_store():
    # nothing free: the two ended sequences' blocks serve the others, to the last one
    args = (16, [17, 32, 5, 0], [-1, 2, -1, 16], None, [0] * 6, 0, [[7, 3, -1], [1, 2, -1], [4, -1, -1], [-1] * 3], 18)
    got = build(*args)
    check_build(*args, got)
    assert got["n_free"] == [1] and got["table"][1] == [1, 2, 4] and got["table"][3][0] == 3 and got["free"][0] == 7
    assert status() == B().OK


@pytest.mark.parametrize("case", ["rows", "blocks", "width", "negative", "free"])
def test_block_tables_refusals_on_the_device(case):
    lens, new, free, n_free, n_rows = [16, 3, 40], [1, 2, -1], [9, 8, 7, 0, 0, 0, 0], 3, 3
    table = [[0, -1, -1], [1, -1, -1], [2, 3, 4]]
    if case == "rows":
        n_rows = 2
    if case == "blocks":
        new, n_free, n_rows = [32, 40, 0], 2, 72
    if case == "width":
        new = [40, 2, -1]
    if case == "negative":
        lens = [-1, 3, 40]
    if case == "free":
        free = free[:4]
    args = (16, lens, new, None, free, n_free, table, n_rows)
    check_build(*args, build(*args))
    assert status() == B().ERR_BAD_INDEX


# ---- norm, rotation, append -------------------------------------------------------------------------------------------------------

def paged(shape, layout, fill=None, gen=None):
    """A store [n_blocks, bs, Hkv, D] in the given order of memory; "gaps": strides with room between tokens, heads and blocks."""
    nb, bs, h, d = shape
    if layout == "head":
        t = torch.empty(nb, h, bs, d, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    elif layout == "gaps":
        t = torch.empty(nb, bs + 1, h + 1, d + 8, dtype=torch.bfloat16, device="cuda")[:, :bs, :h, :d]
    else:
        t = torch.empty(nb, bs, h, d, dtype=torch.bfloat16, device="cuda")
    if fill is not None:
        t.fill_(fill)
    else:
        t.copy_(torch.randn(*shape, generator=gen, device="cuda"))
    return t


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, seed):
    return torch.randn(*shape, generator=gen(seed), device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("n,H,Hkv,D,bs,layout,norm", [(1, 4, 1, 64, 16, "token", False), (3, 5, 5, 128, 32, "gaps", True), (64, 32, 8, 128, 16, "token", False),
                                                      (77, 40, 8, 128, 64, "head", True), (1500, 8, 2, 64, 128, "head", True), (1027, 6, 3, 128, 16, "gaps", False),
                                                      (1203, 5, 5, 128, 32, "token", True), (9, 2, 1, 128, 16, "gaps", True), (1185, 1, 1, 64, 64, "head", False)])
def test_norm_rope_append(n, H, Hkv, D, bs, layout, norm):
    nb = -(-n // bs) + 2
    q, k, v = randn((n, H, D), 1), randn((n, Hkv, D), 2), randn((n, Hkv, D), 3)
    wq, wk = ((1 + 0.1 * randn((D,), 4 + i).float()).to(torch.bfloat16) if norm else None for i in range(2))
    pos = torch.randint(0, 131072, (n,), generator=gen(6), device="cuda", dtype=torch.int32)
    slots = torch.randperm(nb * bs, generator=gen(7), device="cuda")[:n].to(torch.int32)
    if n > 5:
        slots[3] = -1
    k_store, v_store = paged((nb, bs, Hkv, D), layout, -7.0), paged((nb, bs, Hkv, D), layout, -7.0)
    k0, q_out = k.clone(), torch.empty_like(q)
    b = B()
    b.relaxkv_qk_norm_rope_append_paged(b.PagedStore(k_store, v_store), q, k, v, pos, slots, 5.0e5, q_out, wq, wk, 1e-5)
    assert status() == b.OK and torch.equal(k, k0)
    w = lambda x: None if x is None else f64(x)
    theta, p = float(np.float32(5.0e5)), pos.cpu().numpy().astype(np.float64)
    for got, x, weight in ((f64(q_out), q, wq), (None, k, wk)):
        want = orc.norm_rope(f64(x), w(weight), float(np.float32(1e-5)), p, theta)
        if got is None:
            full = f64(k_store)
            s = slots.cpu().numpy()
            got = np.stack([full[x // bs, x % bs] if x >= 0 else orc.to_bf16(want[i]) for i, x in enumerate(s)])
        # one rounding of an fp32 sum of two products, each of the size of the pair's length
        half = D // 2
        length = np.sqrt(want[..., :half] ** 2 + want[..., half:] ** 2)
        assert orc.rounded_within(got, want, 2e-6 * np.concatenate([length, length], -1)).all()
    keep = slots >= 0
    s = slots[keep].long()
    assert torch.equal(v_store[s // bs, s % bs], v[keep])
    rest = torch.ones(nb, bs, dtype=torch.bool, device="cuda")
    rest[s // bs, s % bs] = False
    assert (k_store[rest] == -7).all() and (v_store[rest] == -7).all()
    # in place
    b.relaxkv_qk_norm_rope_append_paged(b.PagedStore(k_store, v_store), q, k, v, pos, slots, 5.0e5, q, wq, wk, 1e-5)
    assert torch.equal(q, q_out)


def test_append_reports_slots_outside_the_store():
    b = B()
    q, k, v = randn((4, 4, 64), 1), randn((4, 1, 64), 2), randn((4, 1, 64), 3)
    ks, vs = paged((3, 16, 1, 64), "token", 5.0), paged((3, 16, 1, 64), "token", 5.0)
    b.relaxkv_qk_norm_rope_append_paged(b.PagedStore(ks, vs), q, k, v, i32([0, 1, 2, 3]), i32([48, -2, 2**31 - 1, 47]), 1e4, torch.empty_like(q))
    assert status() == b.ERR_BAD_INDEX
    assert torch.equal(vs[2, 15], v[3]) and (vs.view(48, -1)[:47] == 5).all() and (ks.view(48, -1)[:47] == 5).all()


# ---- attention ----------------------------------------------------------------------------------------------------------------------

class Step:
    """Contexts in a cache, sequences in a store, the rows of a step.  What belongs to nobody - cache rows between the contexts, the rest of
    a sequence's last block, blocks of no sequence - is NaN; table entries behind a sequence's blocks are out of range."""

    def __init__(self, H, Hkv, D, ctx, seqs, own, new, bs, seed=0, layout="token", ctx_layout="token", bound_slack=0, len_slack=0, q_scale=1.0):
        b = B()
        rng = np.random.default_rng(seed)
        self.H, self.Hkv, self.D, self.ctx, self.bs = H, Hkv, D, list(ctx), bs
        gap = 5
        self.at = [gap + sum(t + gap for t in ctx[:i]) for i in range(len(ctx))]
        total = gap + sum(t + gap for t in ctx)
        self.k, self.v = (self._cache(total, Hkv, D, ctx_layout) for _ in range(2))
        for i, t in enumerate(ctx):
            for j, x in enumerate((self.k, self.v)):
                x[self.at[i]:self.at[i] + t] = randn((t, Hkv, D), 100 * seed + 10 * i + j + 1)
        self.seq_cu = [sum(seqs[:i]) for i in range(len(seqs) + 1)]
        n_seq = self.seq_cu[-1]
        own = own if isinstance(own, list) else [int(x) for x in rng.integers(0, own + 1, n_seq)]      # tokens before the step
        new = new if isinstance(new, list) else [new] * n_seq
        self.row_seq = [i for i in range(n_seq) for _ in range(new[i])]
        self.row_len = [own[i] + j + 1 for i in range(n_seq) for j in range(new[i])]
        have = [-(-(o + n) // bs) for o, n in zip(own, new)]
        nb, width = sum(have) + 3, max(have + [1])
        ids = rng.permutation(nb).tolist()
        self.table = [[ids.pop() for _ in range(h)] + [nb + 7] * (width - h) for h in have]
        self.ks, self.vs = (paged((nb, bs, Hkv, D), layout, float("nan")) for _ in range(2))
        for i in range(n_seq):
            for t in range(own[i] + new[i]):
                self.ks[self.table[i][t // bs], t % bs] = randn((Hkv, D), 7_000_003 * (seed + 1) + 9973 * i + 2 * t)
                self.vs[self.table[i][t // bs], t % bs] = randn((Hkv, D), 7_000_003 * (seed + 1) + 9973 * i + 2 * t + 1)
        n = len(self.row_seq)
        self.q = (q_scale * randn((n, H, D), 55 + seed).float()).to(torch.bfloat16)
        row_cu = [sum(new[:i]) for i in range(n_seq + 1)]
        max_rows = [row_cu[self.seq_cu[i + 1]] - row_cu[self.seq_cu[i]] for i in range(len(ctx))]
        self.max_rows = [min(n, m + bound_slack) for m in max_rows]
        self.max_len = max(self.row_len + [0]) + len_slack
        self.t = dict(row_cu=i32(row_cu), row_seq=i32(self.row_seq), row_len=i32(self.row_len), table=i32(self.table))
        self.shape = b.Shape(H, Hkv, D, ctx)
        self.view = b.CacheView(self.k, self.v, self.at)
        self.store = b.PagedStore(self.ks, self.vs)
        self.out = torch.full((n, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((H, n), 3.0, dtype=torch.float32, device="cuda")

    @staticmethod
    def _cache(total, Hkv, D, layout):
        if layout == "head":
            t = torch.empty(Hkv, total, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        elif layout == "gaps":
            t = torch.empty(total, Hkv + 1, D + 8, dtype=torch.bfloat16, device="cuda")[:, :Hkv, :D]
        else:
            t = torch.empty(total, Hkv, D, dtype=torch.bfloat16, device="cuda")
        return t.fill_(float("nan"))

    def rows(self):
        return B().ContinuationRows(self.seq_cu, self.max_rows, self.max_len, self.t["row_cu"], self.t["row_seq"], self.t["row_len"], self.t["table"])

    def ws(self, block=0):
        return workspace(B().relaxkv_continuation_workspace_bytes(self.shape, len(self.row_seq), block))

    def context_of(self, r):
        return next(b for b in range(len(self.ctx)) if self.seq_cu[b] <= self.row_seq[r] < self.seq_cu[b + 1])

    def shared(self, **kw):
        B().relaxkv_shared_prefix_attention(self.shape, self.view, self.store, self.rows(), self.q, self.out, self.ws(), lse_out=self.lse, **kw)

    def sparse(self, block, lists, **kw):
        B().relaxkv_block_sparse_attention(self.shape, self.view, self.store, self.rows(), block, lists, self.q, self.out, self.ws(), lse_out=self.lse, **kw)

    def keys(self, r, g, block=None, lists=None):
        b = self.context_of(r)
        tok = np.arange(self.ctx[b])
        if lists is not None:
            x = lists[r, g]
            tok = np.concatenate([np.arange(i * block, min((i + 1) * block, self.ctx[b])) for i in x if i >= 0] + [np.zeros(0, dtype=int)]).astype(int)
        out = []
        for c, s in ((self.k64, self.ks64), (self.v64, self.vs64)):
            own = [s[self.table[self.row_seq[r]][t // self.bs], t % self.bs, g] for t in range(self.row_len[r])]
            out.append(np.concatenate([c[self.at[b] + tok, g], np.array(own).reshape(-1, self.D)]))
        return out

    def check(self, block=None, lists=None, skip=()):
        self.k64, self.v64, self.ks64, self.vs64 = f64(self.k), f64(self.v), f64(self.ks), f64(self.vs)
        out, lse, q, G = f64(self.out), f64(self.lse), f64(self.q), self.H // self.Hkv
        for r in range(len(self.row_seq)):
            for g in range(self.Hkv):
                if r in skip:
                    continue
                k, v = self.keys(r, g, block, lists)
                want, want_lse, abs_v, largest = orc.attend(q[r, g * G:(g + 1) * G], k, v, float(np.float32(self.D ** -0.5)))
                got = out[r, g * G:(g + 1) * G]
                assert orc.rounded_within(got, want, orc.attention_delta(abs_v)).all(), (r, g, float(np.abs(got - want).max()))
                got_lse = lse[g * G:(g + 1) * G, r]
                assert ((got_lse == want_lse) | (np.abs(got_lse - want_lse) <= orc.lse_tolerance(largest))).all(), (r, g, got_lse, want_lse)
        assert all((out[r] == 3).all() and (lse[:, r] == 3).all() for r in skip)


ATTEND = {
    "one row, one token": dict(H=4, Hkv=1, D=64, ctx=[1], seqs=[1], own=[0], new=1, bs=16),
    "no context": dict(H=4, Hkv=2, D=128, ctx=[0], seqs=[3], own=[0, 16, 100], new=1, bs=16),
    "some contexts empty": dict(H=8, Hkv=2, D=128, ctx=[0, 300, 0], seqs=[1, 2, 2], own=40, new=1, bs=32, bound_slack=2),
    "sixteen heads": dict(H=32, Hkv=2, D=64, ctx=[500, 129], seqs=[3, 9], own=150, new=1, bs=16, layout="head"),
    "nine heads": dict(H=9, Hkv=1, D=128, ctx=[260], seqs=[15], own=30, new=1, bs=64, ctx_layout="gaps"),
    "five heads, more than a tile of rows": dict(H=10, Hkv=2, D=128, ctx=[1000], seqs=[60], own=70, new=1, bs=16, ctx_layout="head", layout="head"),
    "multi head, gaps": dict(H=3, Hkv=3, D=128, ctx=[128, 127], seqs=[2, 5], own=129, new=1, bs=128, ctx_layout="gaps", layout="gaps"),
    "several tokens each, some none": dict(H=8, Hkv=2, D=128, ctx=[700, 64], seqs=[4, 3], own=100, new=[3, 0, 1, 7, 2, 0, 1], bs=16, len_slack=9),
    "contexts of very different length": dict(H=4, Hkv=1, D=128, ctx=[5000, 100, 1, 2500], seqs=[2, 40, 1, 3], own=300, new=1, bs=32),
    "long own, short context": dict(H=8, Hkv=8, D=64, ctx=[20], seqs=[1], own=[1500], new=1, bs=16),
    "a context nobody continues": dict(H=8, Hkv=2, D=64, ctx=[400, 900], seqs=[0, 2], own=20, new=1, bs=16),
    # (more (row, KV head) pairs than the one-launch form takes)
    "sixteen heads, many rows": dict(H=32, Hkv=2, D=64, ctx=[500, 129], seqs=[10, 15], own=150, new=1, bs=16, layout="head"),
    "nine heads, many rows": dict(H=9, Hkv=1, D=128, ctx=[1260], seqs=[45], own=30, new=1, bs=64, ctx_layout="gaps"),
    "multi head, many rows": dict(H=3, Hkv=3, D=128, ctx=[383, 640], seqs=[12, 5], own=129, new=1, bs=128, ctx_layout="gaps", layout="gaps"),
    "dim 64, long": dict(H=4, Hkv=4, D=64, ctx=[4500], seqs=[12], own=40, new=1, bs=32, ctx_layout="head"),
    "several tokens each, many rows": dict(H=8, Hkv=2, D=128, ctx=[700, 64, 0], seqs=[4, 3, 2], own=100, new=[9, 0, 11, 7, 2, 0, 1, 3, 1], bs=16, len_slack=9, bound_slack=3),
    "sixty pieces": dict(H=2, Hkv=1, D=64, ctx=[16500, 300], seqs=[30, 9], own=90, new=1, bs=16),
    "sixty pieces, wide groups": dict(H=14, Hkv=1, D=128, ctx=[9000], seqs=[60], own=200, new=1, bs=32),
    # (so many (row, KV head) pairs that blocks of one or two consumer warps are taken)
    "a warp per row": dict(H=16, Hkv=8, D=128, ctx=[300, 40], seqs=[70, 45], own=100, new=1, bs=16, ctx_layout="head"),
    "a warp per row, blocks of 128": dict(H=8, Hkv=8, D=64, ctx=[130, 0], seqs=[25, 8], own=200, new=4, bs=128, layout="head"),
    "a warp per row, nine heads": dict(H=18, Hkv=2, D=64, ctx=[70], seqs=[450], own=30, new=1, bs=32),
    "a warp per row, sixteen heads": dict(H=128, Hkv=8, D=128, ctx=[200], seqs=[112], own=20, new=1, bs=16, layout="gaps"),
    "two warps per row": dict(H=8, Hkv=8, D=128, ctx=[500], seqs=[60], own=600, new=1, bs=64, layout="head"),
    "two warps per row, no context": dict(H=48, Hkv=3, D=64, ctx=[0], seqs=[150], own=150, new=1, bs=128),
    "two warps per row, nine heads": dict(H=72, Hkv=8, D=128, ctx=[100], seqs=[57], own=90, new=1, bs=16),
    "large logits, many rows": dict(H=8, Hkv=2, D=128, ctx=[900], seqs=[24], own=60, new=1, bs=16, q_scale=12.0),
    "large logits": dict(H=8, Hkv=2, D=128, ctx=[900], seqs=[4], own=60, new=1, bs=16, q_scale=12.0),
}


@pytest.mark.parametrize("name", list(ATTEND))
def test_shared_prefix_attention(name):
    s = Step(seed=len(name), **ATTEND[name])
    s.shared()
    assert status() == B().OK
    s.check()
    first = s.out.clone()
    s.shared()
    assert torch.equal(first, s.out)


def test_shared_prefix_without_own_tokens_and_rows_without_any_key():
    b = B()
    s = Step(8, 2, 128, [300, 0, 130], [3, 2, 40], [0] * 45, 1, 16, seed=3)
    s.row_len = [0] * 45
    s.t["row_len"], s.max_len = i32(s.row_len), 0
    b.relaxkv_shared_prefix_attention(s.shape, s.view, None, s.rows(), s.q, s.out, s.ws(), lse_out=s.lse)
    assert status() == b.OK
    s.check()
    assert (s.out[3:5] == 0).all() and (s.lse[:, 3:5] == -np.inf).all()
    s = Step(8, 2, 128, [0], [2], [0, 0], 1, 16, seed=3)                 # one sequence without a token, no context
    s.row_len = [0, 1]
    s.t["row_len"] = i32(s.row_len)
    b.relaxkv_shared_prefix_attention(s.shape, None, s.store, s.rows(), s.q, s.out, s.ws(), lse_out=s.lse)
    assert status() == b.OK
    s.check()


def test_one_piece_goes_straight_to_the_output():
    # 128 tokens of context and no own tokens: one slot
    s = Step(16, 16, 64, [100, 90], [5, 9], [0] * 14, 1, 16, seed=4)
    s.row_len = [0] * 14
    s.t["row_len"], s.max_len = i32(s.row_len), 0
    s.shared()
    assert status() == B().OK
    s.check()


@pytest.mark.parametrize("rows", [6, 25])
def test_row_maxima_that_grow_along_the_context(rows):
    s = Step(8, 2, 128, [1500], [rows], 40, 1, 16, seed=5)
    ramp = torch.linspace(0.01, 6.0, 1500, device="cuda")[:, None, None]
    s.k[s.at[0]:s.at[0] + 1500] = (s.k[s.at[0]:s.at[0] + 1500].float() * ramp).to(torch.bfloat16)
    s.shared()
    s.check()


@pytest.mark.parametrize("rows", [2, 50])
def test_infinite_keys_give_their_rows_the_weight_they_ask_for(rows):
    """A key of -inf in a dim where the query is positive has weight zero; where all logits are -inf the row is defined as empty."""
    s = Step(4, 1, 64, [200], [rows], [0, 20] + [1] * (rows - 2), 1, 16, seed=6)
    s.q[:] = s.q.abs() + 0.1
    s.k[s.at[0] + 3:s.at[0] + 9, 0, 5] = float("-inf")
    s.k[s.at[0] + 150:s.at[0] + 200, 0, 7] = float("-inf")
    s.shared()
    s.check()


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("what", ["seq", "len", "bound", "block", "gone"])
def test_shared_prefix_device_refusals(what, many):
    """many: a third context with rows of its own, so that the call takes the prefix kernel."""
    s = Step(8, 2, 128, [300, 200] + [150] * many, [3, 4] + [20] * many, 50, 1, 16, seed=7)
    skip, want = (), B().ERR_BAD_INDEX
    if what == "seq":
        s.t["row_seq"][2] = 7
        skip = (2,)
    elif what == "len":
        s.t["row_len"][4] = s.max_len + 1
        skip = (4,)
    elif what == "bound":
        s.max_rows[1] = 3
        skip = (3, 4, 5, 6)
    elif what == "gone":
        s.t["row_seq"][5] = -1
        skip, want = (5,), B().OK
    else:                                                               # a sequence's block out of range: its tokens are passed over
        i = max(range(7), key=lambda i: s.row_len[i])
        assert s.row_len[i] > 16
        s.t["table"][i, 0] = -3
        s.shared()
        assert status() == want
        r = i
        s.k64, s.v64, s.ks64, s.vs64 = f64(s.k), f64(s.v), f64(s.ks), f64(s.vs)
        q, G = f64(s.q), 4
        for g in range(2):
            k, v = s.keys(r, g)
            n = s.ctx[s.context_of(r)]
            k, v = np.delete(k, slice(n, n + 16), 0), np.delete(v, slice(n, n + 16), 0)
            want_out, _, abs_v, _ = orc.attend(q[r, g * G:(g + 1) * G], k, v, float(np.float32(128 ** -0.5)))
            assert orc.rounded_within(f64(s.out)[r, g * G:(g + 1) * G], want_out, orc.attention_delta(abs_v)).all()
        return
    s.shared()
    assert status() == want
    s.check(skip=skip)


@pytest.mark.parametrize("rows", [5, 30])
def test_other_stream_and_graph(rows):
    s = Step(8, 2, 128, [700], [rows], 90, 1, 16, seed=8)
    s.shared()
    ref = s.out.clone()
    rows, ws, side = s.rows(), s.ws(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: B().relaxkv_shared_prefix_attention(s.shape, s.view, s.store, rows, s.q, s.out, ws, lse_out=s.lse)
    s.out.fill_(3)
    torch.cuda.synchronize()
    B().relaxkv_shared_prefix_attention(s.shape, s.view, s.store, rows, s.q, s.out, ws, stream=side)
    side.synchronize()
    assert torch.equal(ref, s.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    s.out.fill_(3)
    s.q.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    s.check()
    assert not torch.equal(ref, s.out)


@pytest.mark.parametrize("rows", [5, 30])
def test_plain_launches_and_an_expired_wait(rows):
    """The same bits with plain launches; after an expired wait nothing is written until the status word has been read."""
    b = B()
    s = Step(8, 2, 128, [700], [rows], 90, 1, 16, seed=15)
    s.shared()
    ref = s.out.clone()
    before = b.relaxkv_set_chained_launch(False)
    try:
        s.out.fill_(3)
        s.shared()
        assert torch.equal(s.out, ref)
    finally:
        b.relaxkv_set_chained_launch(before)
    s.out.fill_(3)
    b.relaxkv_debug_wait_timeout()
    lists = torch.zeros(rows, 2, 3, dtype=torch.int32, device="cuda")
    lists[:, :, 1], lists[:, :, 2] = 2, -1
    s.shared()
    s.sparse(64, lists)
    torch.cuda.synchronize()
    assert (s.out == 3).all()
    assert status() == b.ERR_TIMEOUT
    s.shared()
    assert torch.equal(s.out, ref) and status() == b.OK


def test_rows_that_their_offsets_do_not_hold():
    """row_cu and row_seq that contradict each other: reported, nothing outside the step's rows is touched."""
    b = B()
    for what in ("end", "elsewhere"):
        s = Step(8, 2, 128, [300, 200], [12, 14], 50, 1, 16, seed=16)
        if what == "end":
            s.t["row_cu"][-1] = 27
        else:
            s.t["row_seq"][3] = 20
        s.max_rows = [26, 26]
        s.shared()
        assert status() == b.ERR_BAD_INDEX
        s.check(skip=tuple(range(12, 26)) if what == "end" else (3,))


# ---- bounds, selection, sparse attention ----------------------------------------------------------------------------------------------

def get_bounds(s, block):
    b = B()
    nb = sum(-(-t // block) for t in s.ctx)
    bounds = torch.full((nb, s.Hkv, 2, s.D), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((nb, s.Hkv), 99.0, device="cuda")
    b.relaxkv_block_bounds(s.shape, b.CacheView(s.k, None, s.at), block, bounds, scale)
    return bounds, scale


def check_bounds(s, block, bounds, scale):
    k, at = f64(s.k), 0
    for i, t in enumerate(s.ctx):
        nb = -(-t // block)
        want, want_scale = orc.bounds(k[s.at[i]:s.at[i] + t], block)
        assert np.array_equal(bounds[at:at + nb].cpu().numpy(), want) and np.array_equal(f64(scale[at:at + nb]), want_scale)
        at += nb


@pytest.mark.parametrize("Hkv,D,ctx,block,layout", [(1, 64, [1], 16, "token"), (2, 128, [100, 0, 64, 33], 16, "token"), (3, 128, [500], 64, "gaps"),
                                                    (8, 64, [257, 128], 128, "head"), (2, 128, [95], 32, "head")])
def test_block_bounds(Hkv, D, ctx, block, layout):
    s = Step(Hkv, Hkv, D, ctx, [1] * len(ctx), 3, 1, 16, seed=9, ctx_layout=layout)
    check_bounds(s, block, *get_bounds(s, block))
    assert status() == B().OK


def test_block_bounds_of_special_values():
    s = Step(2, 2, 64, [96], [1], 3, 1, 16, seed=10)
    k = s.k[s.at[0]:s.at[0] + 96]
    k[:16, 0] = 0.0                                        # all zero: scale 1
    k[:16, 1] = torch.tensor(1.984375 * 2.0 ** 6)          # exactly 127
    k[16:32, 0] = torch.tensor(1.9921875 * 2.0 ** 6)       # just above: 127.5
    k[16:32, 1] = -1.9921875 * 2.0 ** -3
    k[32:48, 0] = 1e-38                                    # below 2^-100 * 127: kept at that scale
    k[32:48, 1, :3] = float("nan")                         # NaN dims count as 0
    k[33, 0, 4] = float("nan")                             # a NaN among numbers is passed over
    k[48:64, 0, 1] = float("inf")                          # clamped
    k[48:64, 0, 2] = float("-inf")
    k[64:80, 1] = 3.3895313892515355e38                    # the largest bf16
    check_bounds(s, 16, *get_bounds(s, 16))


SPARSE = {
    "one block": dict(H=4, Hkv=1, D=64, ctx=[10], seqs=[1], own=[0], new=1, bs=16),
    "few blocks": dict(H=8, Hkv=2, D=128, ctx=[1000, 0, 77], seqs=[3, 2, 2], own=70, new=1, bs=32),
    "five heads": dict(H=10, Hkv=2, D=128, ctx=[3000], seqs=[5], own=40, new=2, bs=16, layout="head", ctx_layout="head"),
    "sixteen heads": dict(H=16, Hkv=1, D=64, ctx=[2000, 2500], seqs=[2, 5], own=40, new=1, bs=128, ctx_layout="gaps"),
    "eight heads": dict(H=8, Hkv=1, D=128, ctx=[4000], seqs=[21], own=20, new=1, bs=16),
    "single heads": dict(H=2, Hkv=2, D=64, ctx=[900], seqs=[3], own=20, new=[1, 0, 3], bs=16, layout="gaps"),
    "two warps per row": dict(H=16, Hkv=8, D=128, ctx=[600, 0], seqs=[50, 10], own=30, new=1, bs=32, ctx_layout="head"),
    "a warp per row": dict(H=8, Hkv=8, D=64, ctx=[400], seqs=[115], own=20, new=1, bs=64, layout="head"),
}


@pytest.mark.parametrize("block,n_select,n_first,n_last", [(16, 5, 1, 2), (64, 7, 0, 1), (32, 64, 2, 0), (128, 3, 0, 0)])
@pytest.mark.parametrize("name", list(SPARSE))
def test_select_and_sparse_attention(name, block, n_select, n_first, n_last):
    b = B()
    s = Step(seed=len(name) + block, **SPARSE[name])
    bounds, scale = get_bounds(s, block)
    check_bounds(s, block, bounds, scale)
    n = len(s.row_seq)
    lists = torch.full((n, s.Hkv, n_select), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, block, bounds, scale, s.rows(), s.q, n_first, n_last, lists, s.ws(block))
    at = np.concatenate([[0], np.cumsum([-(-t // block) for t in s.ctx])])
    bi, sc, q = bounds.cpu().numpy().astype(np.int64), f64(scale), f64(s.q)
    for r in range(n):
        c = s.context_of(r)
        want = orc.select(q[r], bi[at[c]:at[c + 1]], sc[at[c]:at[c + 1]], n_select, n_first, n_last)
        assert np.array_equal(lists[r].cpu().numpy(), want), r
    s.sparse(block, lists)
    assert status() == b.OK
    s.check(block, lists.cpu().numpy())


@pytest.mark.parametrize("n_select,n_first,n_last", [(300, 1, 2), (2, 1, 1), (8700, 0, 3)])
def test_selection_among_very_many_blocks(n_select, n_first, n_last):
    """8750 blocks: more than a block of the launch keeps in shared memory."""
    b = B()
    s = Step(2, 1, 64, [140000], [3], 3, 1, 16, seed=17)
    bounds, scale = get_bounds(s, 16)
    lists = torch.full((3, 1, n_select), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, n_first, n_last, lists, s.ws(16))
    assert status() == b.OK
    bi, sc, q = bounds.cpu().numpy().astype(np.int64), f64(scale), f64(s.q)
    for r in range(3):
        assert np.array_equal(lists[r].cpu().numpy(), orc.select(q[r], bi, sc, n_select, n_first, n_last))


@pytest.mark.parametrize("what", ["bound", "seq", "gone"])
def test_selection_device_refusals(what):
    b = B()
    s = Step(8, 2, 64, [900, 200], [3, 4], 5, 1, 16, seed=18)
    bounds, scale = get_bounds(s, 16)
    good = torch.full((7, 2, 20), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 1, 1, good, s.ws(16))
    lists, skip, want = torch.full_like(good, -9), [2], b.ERR_BAD_INDEX
    if what == "bound":
        s.max_rows[0], skip = 2, [0, 1, 2]
    elif what == "seq":
        s.t["row_seq"][2] = 9
    else:
        s.t["row_seq"][2], want = -1, b.OK
    assert status() == b.OK
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 1, 1, lists, s.ws(16))
    assert status() == want
    keep = [r for r in range(7) if r not in skip]
    assert (lists[skip] == -9).all() and torch.equal(lists[keep], good[keep])


@pytest.mark.parametrize("H,Hkv,D,rows", [(4, 2, 128, [37, 3]), (6, 2, 64, [16, 17]), (10, 2, 128, [8, 19]), (8, 1, 64, [9, 7]), (24, 2, 128, [9, 4]),
                                          (16, 1, 64, [5, 8]), (3, 3, 128, [33, 1])])
def test_selection_for_many_rows(H, Hkv, D, rows):
    """More rows in a context than a block of the launch takes at once, for every way that rows and heads share a product."""
    b = B()
    s = Step(H, Hkv, D, [2100, 1040], rows, 3, 1, 16, seed=19)
    bounds, scale = get_bounds(s, 16)
    n = sum(rows)
    lists = torch.full((n, Hkv, 9), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 1, 2, lists, s.ws(16))
    assert status() == b.OK
    bi, sc, q, first = bounds.cpu().numpy().astype(np.int64), f64(scale), f64(s.q), [0, 132, 197]
    for r in range(n):
        c = 0 if r < rows[0] else 1
        assert np.array_equal(lists[r].cpu().numpy(), orc.select(q[r], bi[first[c]:first[c + 1]], sc[first[c]:first[c + 1]], 9, 1, 2)), r


def test_scores_are_exact_up_to_their_largest_value():
    """Sums of 128 products of 127 x 127 that differ by one part in 16129."""
    b = B()
    s = Step(8, 2, 128, [1600], [3], 5, 1, 16, seed=20)
    k = torch.full((100, 16, 2, 128), 127.0, device="cuda")
    k[..., 5] -= (torch.arange(100, device="cuda") * 37 % 101)[:, None, None].float()
    s.k[s.at[0]:s.at[0] + 1600] = k.reshape(1600, 2, 128).to(torch.bfloat16)
    s.q.fill_(127)
    s.q[1, :, 0] = 1                                         # (a lower score for all blocks)
    s.q[2, :, 5] = 2
    bounds, scale = get_bounds(s, 16)
    lists = torch.empty(3, 2, 40, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 0, 0, lists, s.ws(16))
    want = torch.argsort(torch.arange(100) * 37 % 101, stable=True)[:40].sort().values
    assert (lists.cpu() == want).all()


def test_equal_scores_go_to_the_lower_block():
    b = B()
    s = Step(8, 2, 64, [1600], [2], 5, 1, 16, seed=12)
    s.k[s.at[0]:s.at[0] + 1600] = s.k[s.at[0]:s.at[0] + 16].repeat(100, 1, 1)
    s.k[s.at[0] + 800:s.at[0] + 816] *= 3
    bounds, scale = get_bounds(s, 16)
    lists = torch.empty(2, 2, 6, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 0, 1, lists, s.ws(16))
    assert lists.tolist() == [[[0, 1, 2, 3, 50, 99]] * 2] * 2
    s.q.zero_()                                              # every score is zero
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, 0, 0, lists, s.ws(16))
    assert lists.tolist() == [[[0, 1, 2, 3, 4, 5]] * 2] * 2


def test_sparse_lists_in_any_order_and_bad_entries():
    b = B()
    s = Step(8, 2, 128, [330], [3], 30, 1, 16, seed=13)
    lists = np.array([[[5, -1, 0, 3], [-1, -1, -1, 2]], [[-1] * 4, [1, 0, 4, 5]], [[2, 1, 5, 0]] * 2])
    s.sparse(64, i32(lists))
    assert status() == b.OK
    s.check(64, lists)
    bad = lists.copy()
    bad[2, 0] = [2, 6, 5, -7]
    s.sparse(64, i32(bad))
    assert status() == b.ERR_BAD_INDEX
    bad[2, 0] = [2, -1, 5, -1]
    s.check(64, bad)


def test_rows_of_a_long_cache_lie_behind_32_bit_offsets():
    """A context and a block whose first element is more than 2^31 elements behind the base (9 GB of cache, 5 GB of store)."""
    b = B()
    H, Hkv, D, bs = 8, 2, 128, 16
    tokens = (1 << 31) // (Hkv * D) + 1000
    k = torch.empty(tokens, Hkv, D, dtype=torch.bfloat16, device="cuda")
    s = Step(H, Hkv, D, [300], [2], 40, 1, bs, seed=14)
    at = tokens - 400
    k[at:at + 300] = s.k[s.at[0]:s.at[0] + 300]
    nb = (1 << 31) // (bs * Hkv * D) + 50
    store = torch.empty(nb, bs, Hkv, D, dtype=torch.bfloat16, device="cuda")
    far = [[nb - 1 - x if x < s.ks.shape[0] else nb + 1 for x in row] for row in s.table]
    for row, moved in zip(s.table, far):
        for x, y in zip(row, moved):
            if x < s.ks.shape[0]:
                store[y] = s.ks[x]
    # the same tensors serve as keys and values
    s.v[s.at[0]:s.at[0] + 300] = s.k[s.at[0]:s.at[0] + 300]
    s.vs.copy_(s.ks)
    s.shared()
    s.check()
    ref, ref_lse = s.out.clone(), s.lse.clone()
    s.t["table"] = i32(far)
    rows = b.ContinuationRows(s.seq_cu, s.max_rows, s.max_len, s.t["row_cu"], s.t["row_seq"], s.t["row_len"], s.t["table"])
    view, paged_store = b.CacheView(k, k, [at]), b.PagedStore(store, store)
    b.relaxkv_shared_prefix_attention(s.shape, view, paged_store, rows, s.q, s.out, s.ws(), lse_out=s.lse)
    assert status() == b.OK and torch.equal(s.out, ref) and torch.equal(s.lse, ref_lse)
    lists = i32([[[0, 1, 2, 3, 4]] * Hkv] * 2)
    b.relaxkv_block_sparse_attention(s.shape, view, paged_store, rows, 64, lists, s.q, s.out, s.ws(), lse_out=s.lse)
    s.check()
    slots = i32([(nb - 1) * bs + 3, 7])
    kn = randn((2, Hkv, D), 77)
    b.relaxkv_qk_norm_rope_append_paged(paged_store, s.q, kn, kn, i32([0, 0]), slots, 1e4, torch.empty_like(s.q))
    assert status() == b.OK and torch.equal(store[nb - 1, 3], kn[0]) and torch.equal(store[0, 7], kn[1])
    del k, store
    torch.cuda.empty_cache()
