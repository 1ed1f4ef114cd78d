"""Continuations on the host (no GPU): what the entry points refuse before any launch, how keys are cut into pieces, workspaces."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2609_33503_b200 import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_33503_b200", "csrc")
FAKE, ODD = 0x10000, 0x10008        # never dereferenced: these calls fail before any launch
KEEP = []


def store(**kw):
    v = dict(k=FAKE, v=FAKE, block_stride=16 * 2 * 128, token_stride=2 * 128, head_stride=128, block_size=16, n_blocks=100)
    v.update(kw)
    return B._PagedCache(**v)


def cache(**kw):
    off = (ctypes.c_int64 * 4)(0, 0, 0, 0)
    c = B._CacheView()
    v = dict(k=FAKE, v=FAKE, token_stride=256, head_stride=128)
    v.update(kw)
    for name, x in v.items():
        setattr(c, name, x)
    c.h_req_token_offset = ctypes.cast(off, ctypes.POINTER(ctypes.c_int64))
    KEEP.append(off)
    return c


def rows(seq_cu=(0, 2, 5), max_rows=(2, 3), **kw):
    cu, mr = B._i32(seq_cu), B._i32(max_rows)
    KEEP.extend((cu, mr))
    v = dict(n_seq=seq_cu[-1], table_width=4, table_stride=4, n_rows=5, max_len=60, h_seq_cu=ctypes.addressof(cu), h_max_rows=ctypes.addressof(mr),
             row_cu=FAKE, row_seq=FAKE, row_len=FAKE, block_table=FAKE)
    v.update(kw)
    return B._ContinuationRows(**v)


def shape(ctx=(300, 200), heads=(8, 2), d=128, scale=0.1):
    s = B.Shape(heads[0], heads[1], d, list(ctx), None, scale)
    KEEP.append(s)
    return s


def ref(x):
    KEEP.append(x)                  # (an address keeps nothing alive)
    return None if x is None else ctypes.addressof(x.c if isinstance(x, B.Shape) else x)


BIG = 1 << 40


def attend(s=None, c="", p="", r=None, q=FAKE, out=FAKE, ws=FAKE, nbytes=BIG, entry="relaxkv_shared_prefix_attention", block=64, blocks=FAKE, n_select=8):
    a = [ref(s or shape()), ref(cache() if c == "" else c), ref(store() if p == "" else p), ref(r or rows())]
    if entry == "relaxkv_block_sparse_attention":
        a += [block, blocks, n_select]
    return getattr(B.lib(), entry)(*a, q, out, None, ws, nbytes, 0)


INVALID, SHAPE, SMALL = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED_SHAPE, B.ERR_WORKSPACE_TOO_SMALL
ATTEND = [
    (dict(s=shape(heads=(8, 3))), INVALID), (dict(s=shape(d=96)), SHAPE), (dict(s=shape(heads=(34, 2))), SHAPE), (dict(s=shape(ctx=(-1, 5))), INVALID),
    (dict(s=shape(scale=0.0)), INVALID), (dict(c=None), INVALID), (dict(c=cache(k=ODD)), INVALID), (dict(c=cache(token_stride=257)), INVALID),
    (dict(p=None), INVALID), (dict(p=store(v=None)), INVALID), (dict(p=store(k=ODD)), INVALID), (dict(p=store(block_size=24)), SHAPE),
    (dict(p=store(n_blocks=0)), INVALID), (dict(p=store(n_blocks=1 << 28)), INVALID), (dict(p=store(head_stride=130)), INVALID),
    (dict(p=store(block_stride=64)), INVALID), (dict(r=rows(h_seq_cu=None)), INVALID), (dict(r=rows(seq_cu=(1, 2, 5))), INVALID),
    (dict(r=rows(seq_cu=(0, 6, 5))), INVALID), (dict(r=rows(n_seq=6)), INVALID), (dict(r=rows(max_rows=(-1, 3))), INVALID),
    (dict(r=rows(max_rows=(2, 6))), INVALID), (dict(r=rows(row_cu=None)), INVALID), (dict(r=rows(row_seq=None)), INVALID),
    (dict(r=rows(row_len=None)), INVALID), (dict(r=rows(block_table=None)), INVALID), (dict(r=rows(table_stride=3)), INVALID),
    (dict(r=rows(table_width=0)), INVALID), (dict(r=rows(max_len=-1)), INVALID), (dict(r=rows(n_rows=-1)), INVALID),
    (dict(r=rows(n_rows=1 << 30)), SHAPE), (dict(r=rows(max_len=0x7fffffff)), SHAPE), (dict(s=shape(ctx=(0x7fffffff, 0))), SHAPE), (dict(q=None), INVALID), (dict(q=ODD), INVALID), (dict(out=ODD), INVALID), (dict(ws=None), INVALID),
    (dict(ws=0x10010), INVALID), (dict(nbytes=1000), SMALL),
]


@pytest.mark.parametrize("entry", ["relaxkv_shared_prefix_attention", "relaxkv_block_sparse_attention"])
@pytest.mark.parametrize("i", range(len(ATTEND)))
def test_attention_refusals(entry, i):
    kw, want = ATTEND[i]
    assert attend(entry=entry, **kw) == want


def test_sparse_refusals():
    for kw, want in ((dict(block=48), SHAPE), (dict(blocks=None), INVALID), (dict(n_select=0), INVALID), (dict(n_select=1 << 30), SHAPE)):
        assert attend(entry="relaxkv_block_sparse_attention", **kw) == want
    assert attend(r=rows(n_rows=0, max_rows=(0, 0))) == B.OK                      # nothing to do


def test_block_table_refusals():
    base = dict(n_seq=4, bs=16, seq_len=FAKE, new_len=FAKE + 64, seq_base=None, free=FAKE, cap=10, n_free=FAKE + 128, table=FAKE, width=4, stride=4, n_rows=4,
                len_out=FAKE + 192, free_out=FAKE + 256, cu=FAKE, row_seq=FAKE, row_pos=FAKE, row_len=FAKE, row_slot=FAKE)
    call = lambda **kw: B.lib().relaxkv_build_block_tables(*dict(base, **kw).values(), 0)
    for kw, want in ((dict(n_seq=0), INVALID), (dict(n_seq=4097), SHAPE), (dict(bs=8), SHAPE), (dict(bs=256), SHAPE), (dict(seq_len=None), INVALID),
                     (dict(new_len=None), INVALID), (dict(free=None), INVALID), (dict(cap=-1), INVALID), (dict(n_free=None), INVALID), (dict(table=None), INVALID),
                     (dict(width=0), INVALID), (dict(stride=3), INVALID), (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 31), SHAPE), (dict(len_out=FAKE), INVALID),
                     (dict(len_out=FAKE + 64), INVALID), (dict(free_out=FAKE + 128), INVALID), (dict(row_slot=None), INVALID), (dict(cu=None), INVALID),
                     (dict(width=1 << 30, stride=1 << 30), SHAPE)):
        assert call(**kw) == want, kw


def test_append_refusals():
    def call(p="", q=FAKE, k=FAKE, v=FAKE, n=4, H=8, Hkv=2, D=128, wq=None, wk=None, eps=1e-6, pos=FAKE, slots=FAKE, theta=1e4, q_out=FAKE):
        return B.lib().relaxkv_qk_norm_rope_append_paged(ref(store() if p == "" else p), q, k, v, n, H, Hkv, D, wq, wk, eps, pos, slots, theta, q_out, 0)
    for kw, want in ((dict(p=None), INVALID), (dict(q=ODD), INVALID), (dict(k=None), INVALID), (dict(v=ODD), INVALID), (dict(q_out=None), INVALID), (dict(n=-1), SHAPE),
                     (dict(H=0), SHAPE), (dict(D=80), SHAPE), (dict(wq=FAKE), INVALID), (dict(wq=FAKE, wk=ODD), INVALID), (dict(eps=-1.0), INVALID),
                     (dict(pos=None), INVALID), (dict(slots=None), INVALID), (dict(theta=1.0), INVALID), (dict(p=store(block_size=20)), SHAPE), (dict(n=0), B.OK)):
        assert call(**kw) == want, kw


def test_bounds_and_selection_refusals():
    bounds = lambda s=None, c="", block=64, out=FAKE, scale=FAKE: B.lib().relaxkv_block_bounds(ref(s or shape()), ref(cache() if c == "" else c), block, out, scale, 0)
    for kw, want in ((dict(block=65), SHAPE), (dict(c=None), INVALID), (dict(out=None), INVALID), (dict(out=ODD), INVALID), (dict(scale=None), INVALID),
                     (dict(s=shape(d=32)), SHAPE), (dict(s=shape(ctx=(0, 0)), c=None), B.OK)):
        assert bounds(**kw) == want, kw

    def select(s=None, block=64, b=FAKE, scale=FAKE, r=None, q=FAKE, n=8, first=1, last=2, out=FAKE, ws=FAKE, nbytes=BIG):
        return B.lib().relaxkv_select_blocks(ref(s or shape()), block, b, scale, ref(r or rows()), q, n, first, last, out, ws, nbytes, 0)
    for kw, want in ((dict(block=0), SHAPE), (dict(n=0), INVALID), (dict(first=-1), INVALID), (dict(last=-1), INVALID), (dict(first=5, last=4), INVALID),
                     (dict(b=None), INVALID), (dict(scale=None), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(ws=0x10020), INVALID),
                     (dict(nbytes=64), SMALL), (dict(r=rows(row_len=None, block_table=None, row_seq=None)), INVALID)):
        assert select(**kw) == want, kw


def test_workspace_grows_with_rows_and_contexts():
    rng = random.Random(5)
    size = lambda ctx, n, block: B.relaxkv_continuation_workspace_bytes(B.Shape(32, 8, 128, ctx), n, block)
    for _ in range(500):
        ctx = [rng.randint(0, 70000) for _ in range(rng.randint(1, 8))]
        n, block = rng.randint(0, 3000), rng.choice([0, 16, 64])
        less = [rng.randint(0, t) for t in ctx]
        assert 0 < size(less, n, block) <= size(ctx, n, block)
        assert size(ctx, n, 0) <= size(ctx, n, 16)
    # fewer rows have more slots each: never more room than 4096 row-slots take, or four of every row
    assert size([1000], 1, 0) <= size([1000], 4096, 0)
    assert size([10], 5, 30) == size([-1], 5, 0) == size([10], -1, 0) == 0


MAIN = r"""
#include "continuation_splits.cuh"
#include <cmath>
#include <cstdio>
#include <random>
using namespace relaxkv;
int main() {
  std::mt19937 r(1);
  double worst = 0;
  for (int it = 0; it < 40000; ++it) {
    const int heads = 1 << (r() % 5), n = 1 + r() % 12, sms = 148, most = 4 + r() % 60;
    int tiles[12], rows[12];
    long long all = 0;
    int longest = 0;
    for (int i = 0; i < n; ++i) {
      tiles[i] = (int)std::pow(2.0, std::uniform_real_distribution<>(0, 10)(r));
      rows[i] = it % 3 ? 1 + r() % 3 : r() % 2;
      all += (long long)tiles[i] * rows[i] * heads;
      if (rows[i] && tiles[i] > longest) longest = tiles[i];
    }
    if (!longest) continue;
    const int per = prefix_tiles_per_block(tiles, rows, n, heads, sms, most, 0.01);
    if (per < 1 || (longest + per - 1) / per > most || (per < 2 && longest > 1)) { std::printf("%d tiles per block of %d\n", per, longest); return 1; }
    long long blocks = 0, busy = 0;
    for (int i = 0; i < n; ++i) {
      const long long k = (long long)rows[i] * heads, p = (tiles[i] + per - 1) / per;
      blocks += k * p;
      busy += k * (3 * p + tiles[i]);
    }
    const double best = std::max({(double)(all + 3.0 * heads) / sms, 5.0, (longest + most - 1) / most + 3.0});
    const double took = blocks <= sms ? 3.0 + per : std::max(3.0 + per, (double)busy / sms + 0.5 * (3 + per));
    worst = std::max(worst, took / best);
  }
  if (worst > 6.0) { std::printf("%.2f times the best\n", worst); return 1; }
  for (int it = 0; it < 40000; ++it) {
    const long long items = 1 + (long long)std::pow(2.0, std::uniform_real_distribution<>(0, 16)(r)), tiles = 1 + r() % 5000;
    const int most = 1 + r() % 64, p = paged_pieces(items, tiles, 148, most), c = paged_cluster(items, tiles, 148, 8);
    if (p < 1 || p > most || (p > 1 && (tiles + 1) / 2 < p)) { std::printf("%lld items of %lld tiles: %d pieces\n", items, tiles, p); return 1; }
    if (c < 0 || c > 8 || (c > 1 && (tiles + 1) / 2 < c)) { std::printf("%lld items of %lld tiles: a cluster of %d\n", items, tiles, c); return 1; }
    if (items >= 296 && c != 1) { std::printf("%lld items: a cluster of %d\n", items, c); return 1; }
  }
  return 0;
}
"""


def test_how_keys_are_cut(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_the_room_of_a_step_holds_every_smaller_one():
    s, before = B.Shape(4, 2, 64, [1000]), 0
    for n in list(range(0, 1200)) + [4095, 4096, 4097, 20000]:
        nbytes = B.relaxkv_continuation_workspace_bytes(s, n, 0)
        assert nbytes >= before, n
        before = nbytes
