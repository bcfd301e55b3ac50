"""The paged cache on the GPU (ff.paged_append, ff.paged_attention) against the float64
reference of paged_ref.py: types, head layouts, lengths, strides, holes, stale memory, rows of
no sequence, both operators together, streams and graphs."""
from __future__ import annotations

import math
import random

import numpy as np
import pytest
import torch

from paper_2609_32540_amd import ff

import paged_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = torch.device("cuda", 0)


def forms():
    """The forms of this thread's last call: rows of the tiles of few rows (0: not launched), whether
    their keys could be cut, the same of many rows."""
    return tuple(ff.lib().ff_internal_last_paged(i) for i in range(4))


class Case:
    """A pool, a batch and tensors.  news, lens: new tokens and lengths of the sequences; unused
    pool memory holds `stale` (NaN by default)."""

    def __init__(self, news, lens, *, dtype=BF16, d=128, hk=2, group=4, page=16, pad=0, spare=2,
                 stale=math.nan, columns=None, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.page = dtype, page
        cols = columns or max(1, max((-(-n // page) for n in lens), default=1))
        held = [min(-(-max(n, 0) // page), cols) for n in lens]
        self.n_pages = sum(held) + spare
        order = torch.randperm(self.n_pages, generator=g)
        table = torch.full((len(lens), cols), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(held):
            table[s, :n] = order[at:at + n].to(torch.int32)
            at += n
        starts = [0]
        for n in news:
            starts.append(starts[-1] + n)
        self.rows = starts[-1] + pad
        self.b = ref.Batch(starts, list(lens), table, page, self.n_pages)
        self.k_pages = torch.full((self.n_pages, hk, page, d), stale, dtype=dtype)
        self.v_pages = torch.full((self.n_pages, hk, page, d), stale, dtype=dtype)
        for s, n in enumerate(lens):
            for c in range(held[s]):
                m = min(page, n - c * page)
                for pool in (self.k_pages, self.v_pages):
                    pool[int(table[s, c]), :, :m] = torch.randn((hk, m, d), generator=g).to(dtype)
        self.q = torch.randn((self.rows, hk * group, d), generator=g).to(dtype)
        self.g = g

    def on_gpu(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        return (self.k_pages.to(DEV), self.v_pages.to(DEV), torch.tensor(self.b.q_start, **i32),
                torch.tensor(self.b.kv_len, **i32), self.b.table.to(DEV))

    def check_attention(self, q=None, scale=None, rows=None, heads=None, form=None, **kw):
        """Run without and with the log-sum-exp (bf16 prompts then run another pass) and compare; rows
        of no sequence have to keep what `out` held."""
        kp, vp, qs, kl, tb = self.on_gpu()
        q = q if q is not None else self.q.to(DEV)
        hints = {k: kw.pop(k) for k in ("min_new", "max_new") if k in kw}
        call = {k: v for k, v in kw.items() if k != "anchors"}
        r = ref.attention(self.b, self.q, self.k_pages, self.v_pages, scale=scale, rows=rows, heads=heads, **kw)
        mine = r.rows if rows is None else [x for x in r.rows if x in rows]
        others = [x for x in range(self.rows) if x not in set(r.rows)]
        hh = list(range(self.q.shape[1])) if heads is None else list(heads)

        def near(got, exact, tol):
            assert (got[others] == 7.0).all(), "a row of no sequence was written"
            a, e, t = (x[mine][:, hh] for x in (got, exact, tol))
            fine = np.isfinite(e)
            assert np.array_equal(a[~fine], e[~fine], equal_nan=True), "not finite in other places, or another value"
            off = np.abs(a[fine] - e[fine]) - t[fine]
            assert off.size == 0 or off.max() <= 0, f"off by {off.max()} over the bound"

        for lse in (None, torch.full(self.q.shape[:2], 7.0, dtype=F32, device=DEV)):
            out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device=DEV)
            ff.paged_attention(q, kp, vp, qs, kl, tb, out=out, lse=lse, scale=scale,
                               anchor_tokens=kw.get("anchors", 0), **hints, **call)
            if form is not None and self.dtype == BF16:
                assert forms() == form
            near(ref.f64(out), r.out, r.tol)
            if lse is not None:
                near(ref.f64(lse), r.lse, r.lse_tol)


# ---- attention: one new token ------------------------------------------------------
LENS = [1, 0, 2, 15, 16, 17, 31, 32, 33, 64, 100, 255, 256, 257, 700]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,group", [(2, 4), (3, 1), (1, 7), (1, 16), (2, 19)])
def test_decode_lengths(dtype, d, hk, group):
    news = [min(n, 1) for n in LENS]
    Case(news, LENS, dtype=dtype, d=d, hk=hk, group=group).check_attention(max_new=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [31, 71, 300])
@pytest.mark.parametrize("news", [[1, 1, 1], [1, 5, 2]])
def test_one_kv_head_for_many_query_heads(dtype, group, news):
    """A token's heads in several tiles, tiles that begin inside a token."""
    for window in (-1, 100):
        Case(news, [900, 20, 300], dtype=dtype, d=64, hk=1, group=group).check_attention(window=window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_decode_page_sizes(dtype, page):
    Case([1, 1, 1], [page - 1, 3 * page + 5, 611], dtype=dtype, page=page).check_attention(max_new=1)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("lens", [[9001], [5000, 40, 12000], [3000] * 5])
def test_decode_split_over_the_length(dtype, d, lens):
    """Caches long enough for several parts, joined; a short sequence beside long ones."""
    Case([1] * len(lens), lens, dtype=dtype, d=d, hk=1, group=2).check_attention(max_new=1)


def test_decode_many_sequences():
    """More sequences than lanes; some without new tokens."""
    rng = random.Random(5)
    lens = [rng.randint(0, 90) for _ in range(333)]
    news = [min(n, rng.randint(0, 1)) for n in lens]
    Case(news, lens, hk=1, group=2, d=64).check_attention(max_new=1)


def test_decode_most_sequences():
    rng = random.Random(6)
    lens = [rng.randint(1, 40) for _ in range(1024)]
    Case([1] * 1024, lens, hk=2, group=1, d=64).check_attention(max_new=1)


# ---- attention: several new tokens -------------------------------------------------
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("window,anchors", [(-1, 0), (0, 0), (1, 0), (37, 0), (37, 5), (100, 70), (3, 400), (5000, 10)])
def test_several_new_tokens(dtype, d, block, window, anchors):
    news, lens = [3, 0, 1, 40, 17, 5], [200, 50, 33, 40, 333, 5]
    Case(news, lens, dtype=dtype, d=d, hk=2, group=3).check_attention(block=block, window=window, anchors=anchors)


# Small launches of many rows run on the kernel of few rows (tiles of 16 or 32), so what is said
# of the 256-row one is tested at many heads, a few of them checked.
FEW, MANY, BOTH = (32, 0, 0, 0), (0, 0, 256, 0), (32, 1, 256, 0)


@pytest.mark.parametrize("dtype,d,group,hk", [(BF16, 128, 4, 2), (BF16, 64, 1, 3), (BF16, 128, 1, 1), (F32, 128, 2, 1)])
@pytest.mark.parametrize("block", [False, True])
def test_small_prompts(dtype, d, group, hk, block):
    """Prompts of several tiles, ragged, the first one starting at key 0; sampled rows."""
    news, lens = [700, 129, 1, 64], [700, 400, 350, 77]
    c = Case(news, lens, dtype=dtype, d=d, group=group, hk=hk)
    rows = sorted(set(list(range(0, 700, 37)) + [0, 1, 63, 64, 255, 256, 699, 700, 701, 828, 829, 830, 893]))
    c.check_attention(block=block, rows=rows, form=FEW)


@pytest.mark.parametrize("d,group,hk", [(128, 4, 16), (128, 1, 40), (64, 3, 30), (64, 1, 64)])
@pytest.mark.parametrize("block", [False, True])
def test_prompts(d, group, hk, block):
    """The same on the 256-row kernel, beside a sequence of one new token."""
    news, lens = [900, 300, 1, 70, 0], [900, 1100, 950, 77, 30]
    c = Case(news, lens, d=d, group=group, hk=hk)
    rows = [0, 1, 31, 32, 63, 64, 65, 85, 255, 256, 257, 640, 899, 900, 901, 1199, 1200, 1201, 1202, 1270]
    c.check_attention(block=block, rows=rows, heads=[0, hk * group - 1], form=BOTH)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("kw", [dict(window=0), dict(window=1), dict(window=50, anchors=3), dict(window=300, anchors=130),
                                dict(window=2000, anchors=5), dict(window=50, anchors=3, block=True),
                                dict(window=700, block=True), dict(window=0, block=True)])
def test_prompts_with_windows(d, kw):
    news, lens = [600, 70, 1013], [1200, 500, 1013]
    rows = [0, 1, 31, 32, 127, 128, 255, 256, 599, 600, 601, 669, 670, 671, 700, 800, 925, 926, 1682]
    Case(news, lens, d=d, hk=64, group=1).check_attention(rows=rows, heads=[0, 63], form=MANY, min_new=70, **kw)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("kw", [dict(window=0), dict(window=50, anchors=3), dict(window=300, anchors=130),
                                dict(window=50, anchors=3, block=True), dict(window=700, block=True)])
def test_small_prompts_with_windows(dtype, d, kw):
    news, lens = [300, 70, 513], [900, 500, 513]
    rows = sorted(set(list(range(0, 883, 29)) + [0, 1, 255, 256, 299, 300, 369, 370, 371, 625, 626, 882]))
    Case(news, lens, dtype=dtype, d=d, hk=1, group=2).check_attention(rows=rows, form=FEW, **kw)


@pytest.mark.parametrize("d,hk,news,lens", [(128, 4, [1000], [16000]), (64, 6, [300, 700], [18000, 17000]), (128, 8, [90, 600], [5000, 9100])])
def test_prompts_split_over_the_length(d, hk, news, lens):
    """Few tiles over long caches: their keys in parts."""
    rows = [0, 1, 31, 32, 63, 64, 85, 86, 89, sum(news) // 2, sum(news) - 1]
    for block in (False, True):
        c = Case(news, lens, d=d, hk=hk, group=1, page=64)
        c.check_attention(rows=rows, heads=[0, hk - 1], block=block, min_new=90, form=(0, 0, 256, 1))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_small_prompts_split_over_the_length(dtype, d):
    for block in (False, True):
        c = Case([90, 200], [5000, 3100], dtype=dtype, d=d, hk=1, group=3, page=64)
        c.check_attention(rows=[0, 31, 32, 89, 90, 200, 289], block=block, form=(32, 1, 0, 0))


def test_prompts_past_64_tiles():
    """More key tiles than a wave holds pages of, in one part, with holes."""
    c = Case([1280], [70 * 64 + 5], hk=64, group=1, d=64)
    for col in (0, 3, 100, 255, 256, 257, 270):
        c.b.table[0, col] = -1
    rows = [0, 100, 255, 256, 279, 1279]
    c.check_attention(rows=rows, heads=[0, 63], min_new=1280, form=MANY)
    c.check_attention(rows=rows, heads=[0, 63], block=True, min_new=1280, form=MANY)


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1])
def test_prompts_with_holes(bad):
    """At the start, inside, everywhere; stale memory behind the end."""
    c = Case([600, 500, 300], [900, 1000, 300], hk=64, group=1, d=64)
    c.b.table[0, 0] = c.b.table[0, 5] = bad
    c.b.table[1, 30:40] = bad
    c.b.table[2, :] = bad
    rows = [0, 1, 300, 599, 600, 700, 1099, 1100, 1399]
    for kw in (dict(), dict(block=True, window=160, anchors=20)):
        c.check_attention(rows=rows, heads=[0, 63], min_new=300, form=MANY, **kw)


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_prompt_tokens_that_are_not_finite(value):
    """Causal: V (then K) of one token is not finite, the rows before it are whole."""
    news, length, hk = 700, 1000, 64
    for which in ("v", "k"):
        c = Case([news], [length], d=64, hk=hk, group=1)
        j = length - news + 333
        p, s = c.b.place(0, j)
        if which == "v":
            c.v_pages[p, :, s, 3] = value
        else:
            c.k_pages[p, :, s] = value
        rows = [0, 255, 256, 300, 332] + ([333, 340, 699] if which == "v" else [])
        c.check_attention(rows=rows, heads=[0, 40], min_new=news, form=MANY)


def test_prompt_scores_far_apart():
    """The reference of the first block is left far behind: the checked pass, in parts and whole."""
    for news, length, hk, form in ((1000, 1100, 64, MANY), (256, 24000, 4, (0, 0, 256, 1))):
        c = Case([news], [length], d=128, hk=hk, group=1, page=64)
        for col in range(c.b.table.shape[1]):
            c.k_pages[int(c.b.table[0, col])] *= 1.0 + 3.0 * col * 64 / length * 20
        for block in (False, True):
            c.check_attention(rows=[0, 40, 255, news - 1], heads=[0, hk - 1], block=block, min_new=news, form=form)


@pytest.mark.parametrize("hints", [dict(min_new=0, max_new=1), dict(min_new=64, max_new=64), dict(min_new=500, max_new=0)])
def test_hints_do_not_change_what_is_computed(hints):
    """min_new and max_new that do not hold."""
    Case([150, 1, 30], [150, 900, 300], hk=1, group=2).check_attention(**hints)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_new_tokens_than_the_sequence_holds(dtype):
    """Tokens with an index below 0 see nothing (causal) or the whole sequence (block)."""
    for block in (False, True):
        Case([9, 4, 3], [5, 0, -3], dtype=dtype).check_attention(block=block)


# ---- masked places -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "num_pages"])
def test_holes(dtype, bad):
    """Table entries that name no page: at the start, inside, at the end, everywhere."""
    c = Case([1, 2, 40, 3], [300, 100, 300, 64], dtype=dtype)
    bad = c.n_pages if bad == "num_pages" else bad
    c.b.table[0, 0] = c.b.table[0, 5] = c.b.table[1, 6] = bad
    c.b.table[2, 3:9] = bad
    c.b.table[3, :] = bad
    for kw in (dict(), dict(block=True, window=60, anchors=20)):
        c.check_attention(**kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sequences_longer_than_the_table(dtype):
    c = Case([1, 3, 20], [100, 400, 130], dtype=dtype, columns=5)
    c.check_attention()
    c.check_attention(block=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("length", [100000, 2 ** 31 - 1])
@pytest.mark.parametrize("held", [300, 320])
def test_lengths_far_behind_the_table(dtype, length, held):
    """Every key of the table is before the window: only the anchors are seen, and no block is
    worked on that the table does not hold.  (300 tokens end inside a page, whose stale rest then
    counts as tokens: NaN.)"""
    for news in (2, 90):
        c = Case([news], [held], dtype=dtype, hk=1, group=1, d=64)
        c.b.kv_len[0] = length
        kp, vp, qs, kl, tb = c.on_gpu()
        out = torch.full_like(c.q, 7.0, device=DEV)
        for anchors in (2 ** 31 - 1, 20, 0):
            ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb, window=5, anchor_tokens=anchors, out=out)
            near = ref.Batch([0, news], [400 + news], c.b.table, c.page, c.n_pages)   # as far behind it
            r = ref.attention(near, c.q, c.k_pages, c.v_pages, window=5, anchors=min(anchors, 400))
            got, nan = ref.f64(out), np.isnan(r.out)
            assert (np.isnan(got) == nan).all() and nan.all() == (held == 300 and anchors > 300)
            assert (np.abs(got - r.out)[~nan] <= r.tol[~nan]).all()


@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("news,lens", [([1], [90]), ([5], [90]), ([300], [500])])
def test_an_infinite_value_that_rows_see(block, news, lens):
    """V holds an infinity: the columns that see it are infinite, the others are whole."""
    c = Case(news, lens, d=64, hk=1, group=2)
    for j, col in ((3, 5), (40, 6)):
        p, s = c.b.place(0, j)
        c.v_pages[p, :, s, col] = math.inf
    c.check_attention(block=block, rows=[x for x in (0, 1, 4, 150, 299) if x < news[0]])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("news", [[1], [9], [70]])
def test_masked_memory_does_not_matter(dtype, value, news):
    """What no row sees: behind the end, before the window, pages of nobody."""
    c = Case(news, [170], dtype=dtype, stale=value)
    for j in range(10, 50):
        p, s = c.b.place(0, j)
        c.k_pages[p, :, s] = value
        c.v_pages[p, :, s] = value
    c.check_attention(window=170 - news[0] - 50, anchors=10, block=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("news,length", [(6, 40), (40, 40), (150, 300)])
def test_a_token_that_is_not_finite_reaches_only_the_rows_that_see_it(dtype, value, news, length):
    c = Case([news], [length], dtype=dtype, d=64, hk=1, group=3)
    j = length - news + news // 2
    p, s = c.b.place(0, j)
    c.v_pages[p, :, s, 3] = value
    r = ref.attention(c.b, c.q, c.k_pages, c.v_pages)
    kp, vp, qs, kl, tb = c.on_gpu()
    got = ref.f64(ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb))
    for row, _, i in c.b.tokens(c.rows):
        if i < j:
            assert (np.abs(got[row] - r.out[row]) <= r.tol[row]).all()
        else:
            assert not np.isfinite(got[row, :, 3]).any()
            keep = [x for x in range(64) if x != 3]
            assert (np.abs(got[row][:, keep] - r.out[row][:, keep]) <= r.tol[row][:, keep]).all()
    # a key that is not finite: rows before it are whole
    c = Case([news], [length], dtype=dtype, d=64, hk=1, group=3)
    c.k_pages[p, :, s] = value
    r = ref.attention(c.b, c.q, c.k_pages, c.v_pages, rows=[x for x, _, i in c.b.tokens(c.rows) if i < j])
    kp, vp, qs, kl, tb = c.on_gpu()
    got = ref.f64(ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb))
    for row, _, i in c.b.tokens(c.rows):
        if i < j:
            assert (np.abs(got[row] - r.out[row]) <= r.tol[row]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_far_apart(dtype):
    """Keys whose scores rise along the cache (the reference moves) and a row of one loud key."""
    c = Case([1, 4, 90, 300], [900, 500, 200, 800], dtype=dtype, hk=1, group=2)
    for s in range(4):
        for j in range(c.b.kv_len[s]):
            p, sl = c.b.place(s, j)
            c.k_pages[p, :, sl] *= 1.0 + j / 20.0
    c.check_attention(rows=[0, 1, 4, 5, 30, 94, 95, 200, 394])
    c.check_attention(rows=[0, 94, 394], block=True)


@pytest.mark.parametrize("dtype,news,length,hk,form", [
    (BF16, [1, 1], 700, 1, None), (BF16, [1], 9000, 1, None), (BF16, [20], 300, 1, None), (BF16, [700], 1000, 64, MANY),
    (F32, [1, 1], 700, 1, None), (F32, [1], 9000, 1, None), (F32, [20], 300, 1, None)])
def test_large_values_under_rising_scores(dtype, news, length, hk, form):
    """V of 2^100 where scores end 43 log2 units above the first block's: a weight relative to that
    block times V is past float32, the result is not."""
    c = Case(news, [length] * len(news), dtype=dtype, d=64, hk=hk, group=1, page=64)
    c.q[:, :, 0] = 8.0
    for s in range(len(news)):
        for j in range(length):
            p, sl = c.b.place(s, j)
            c.k_pages[p, :, sl, 0] = 30.0 * j / length
    c.v_pages *= 2.0 ** 100
    c.check_attention(rows=[0, sum(news) - 1], heads=[0, hk - 1], max_new=news[0], min_new=news[0], form=form)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_minus_infinity_weigh_nothing(dtype):
    c = Case([1, 20], [100, 60], dtype=dtype, hk=1, group=1, d=64)
    c.q[:, :, 0] = 1.0
    for s, j in ((0, 0), (0, 1), (0, 40), (1, 0), (1, 2), (1, 45)):
        p, sl = c.b.place(s, j)
        c.k_pages[p, :, sl, 0] = -math.inf
    # row 0 of sequence 1 (index 40) and all others still see finite keys
    kp, vp, qs, kl, tb = c.on_gpu()
    got = ref.f64(ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb))
    holes = c.k_pages.clone()
    holes[holes == -math.inf] = -1e4     # weight exp(-1000): nothing, in float64 as well
    r = ref.attention(c.b, c.q, holes, c.v_pages)
    e = np.abs(got - r.out)
    u = ref.U_BF16 if dtype == BF16 else 300 * ref.U_F32
    assert (e <= 2.1 * u * (np.abs(r.out) + 4.0)).all()


# ---- layout ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_no_sequence_strides_and_tables(dtype):
    c = Case([2, 1, 30], [50, 20, 40], dtype=dtype, hk=2, group=2, d=64, pad=5)
    wide = torch.randn((c.rows, 4 + 3, 64), generator=c.g).to(dtype).to(DEV)
    wide[:, 2:6] = c.q.to(DEV)
    c.check_attention(q=wide[:, 2:6])
    # a table that is a slice of a wider one
    kp, vp, qs, kl, tb = c.on_gpu()
    big = torch.full((3, tb.shape[1] + 9), 12345, dtype=torch.int32, device=DEV)
    big[:, 4:4 + tb.shape[1]] = tb
    a = ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, big[:, 4:4 + tb.shape[1]])
    b = ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb)
    n = c.b.q_start[-1]
    assert torch.equal(a[:n], b[:n])


def test_rows_before_the_first_sequence():
    c = Case([3, 2], [30, 40])
    c.b.q_start[:] = [4, 7, 9]
    c.rows = 12
    c.q = torch.randn((12, 8, 128), generator=c.g).to(BF16)
    c.check_attention()


def test_nothing_to_do():
    c = Case([1], [10])
    kp, vp, qs, kl, tb = c.on_gpu()
    q = c.q.to(DEV)
    assert ff.paged_attention(q[:0], kp, vp, qs * 0, kl, tb).shape == (0, 8, 128)
    out = torch.full_like(q, 3.0)
    ff.paged_attention(q, kp, vp, qs[:1], kl[:0], tb[:0], out=out)
    assert (out == 3.0).all()
    ff.paged_attention(q, kp, vp, qs * 0, kl, tb, out=out)      # no new token in any sequence
    assert (out == 3.0).all()


def test_offsets_past_32_bits():
    """Pools of more than 2^32 elements, the sequence's pages at both ends."""
    hk, page, d = 8, 256, 128
    n_pages = 2 ** 32 // (hk * page * d) + 40
    kp = torch.empty((n_pages, hk, page, d), dtype=BF16, device=DEV)
    vp = torch.empty_like(kp)
    length = 1100
    pages = [n_pages - 1, 3, n_pages - 7, 0, n_pages - 2]
    small = Case([1], [length], hk=hk, group=1, page=page)
    for c, p in enumerate(pages):
        at = int(small.b.table[0, c])
        kp[p] = small.k_pages[at].to(DEV)
        vp[p] = small.v_pages[at].to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    qs, kl, tb = torch.tensor([0, 1], **i32), torch.tensor([length], **i32), torch.tensor([pages], **i32)
    got = ref.f64(ff.paged_attention(small.q.to(DEV), kp, vp, qs, kl, tb))
    r = ref.attention(small.b, small.q, small.k_pages, small.v_pages)
    assert (np.abs(got - r.out) <= r.tol).all()
    k = torch.randn((1, hk, d), generator=small.g).to(BF16).to(DEV)
    ff.paged_append(k, k, kp, vp, qs, kl, tb)
    at = (length - 1) % page
    assert torch.equal(vp[pages[4], :, at], k[0])
    want = ref.rotate(ref.f64(k[0]), [length - 1] * 3, ref.rope_split(d), 10000.0)
    assert (np.abs(ref.f64(kp[pages[4], :, at]) - want) <= ref.U_BF16 * np.abs(want) + 1e-9).all()


@pytest.mark.parametrize("dtype,news,group", [(BF16, 600, 4), (F32, 1, 2)])
def test_offsets_past_32_bits_of_the_other_kernels(dtype, news, group):
    hk, page, d, length = 16, 256, 128, 1100
    n_pages = 2 ** 32 // (hk * page * d) + 40
    kp = torch.empty((n_pages, hk, page, d), dtype=dtype, device=DEV)
    vp = torch.empty_like(kp)
    pages = [n_pages - 1, 3, n_pages - 7, 0, n_pages - 2]
    small = Case([news], [length], dtype=dtype, hk=hk, group=group, page=page)
    for c, p in enumerate(pages):
        at = int(small.b.table[0, c])
        kp[p] = small.k_pages[at].to(DEV)
        vp[p] = small.v_pages[at].to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    qs, kl, tb = torch.tensor([0, news], **i32), torch.tensor([length], **i32), torch.tensor([pages], **i32)
    rows, heads = [0, news // 2, news - 1], [0, hk * group - 1]
    got = ref.f64(ff.paged_attention(small.q.to(DEV), kp, vp, qs, kl, tb, min_new=news))
    assert dtype == F32 or forms()[2] == 256
    r = ref.attention(small.b, small.q, small.k_pages, small.v_pages, rows=rows, heads=heads)
    assert (np.abs(got - r.out) <= r.tol)[rows][:, heads].all()


# ---- append ------------------------------------------------------------------------
def check_append(c: Case, hq, *, positions=None, pairs=None, theta=10000.0, wide=False, with_q=True, in_place=False):
    d, hk = c.k_pages.shape[3], c.k_pages.shape[1]
    kp, vp, qs, kl, tb = c.on_gpu()
    k, v = (torch.randn((c.rows, hk, d), generator=c.g).to(c.dtype) for _ in range(2))
    q = torch.randn((c.rows, hq, d), generator=c.g).to(c.dtype)
    if wide:
        x = torch.cat([q, k, v], 1).to(DEV)
        qd, kd, vd = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    else:
        qd, kd, vd = q.to(DEV), k.to(DEV), v.to(DEV)
    q_out = None
    if with_q:
        q_out = qd if in_place else torch.full_like(q, 5.0, device=DEV)
    pos = torch.tensor(positions, dtype=torch.int32) if positions is not None else None
    before = q if in_place else torch.full_like(q, 5.0)
    res = ff.paged_append(kd, vd, kp, vp, qs, kl, tb, q=qd if with_q else None, q_out=q_out,
                          positions=pos.to(DEV) if pos is not None else None, rope_pairs=pairs, rope_theta=theta)
    ek, ev, eq = ref.append(c.b, k, v, c.k_pages, c.v_pages, q if with_q else None, before, positions, pairs, theta)
    u = ref.U_BF16 if c.dtype == BF16 else ref.U_F32
    tiny = 1e-12 * 10      # float64 angles of positions up to 1e5, times values of a few
    written_k = ~np.isclose(ek, ref.f64(c.k_pages), rtol=0, atol=0, equal_nan=True)
    gk, gv = ref.f64(kp), ref.f64(vp)
    same = ~written_k
    assert np.array_equal(gk[same], ref.f64(c.k_pages)[same], equal_nan=True)
    assert (np.abs(gk - ek)[written_k] <= (u * np.abs(ek) + tiny + 1e-38)[written_k]).all()
    assert np.array_equal(gv, ev, equal_nan=True)
    if with_q:
        gq = ref.f64(res)
        assert (np.abs(gq - eq) <= u * np.abs(eq) + tiny).all()
    else:
        assert res is None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,group,page", [(2, 4, 16), (1, 1, 32), (5, 3, 64), (8, 8, 256)])
def test_append(dtype, d, hk, group, page):
    news, lens = [1, 0, 7, 1, 33, 20], [1, 5, 7, 130, 60, 21]
    check_append(Case(news, lens, dtype=dtype, d=d, hk=hk, group=group, page=page, pad=3), hk * group)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_positions_pairs_and_rows(dtype):
    news, lens = [4, 9], [300, 9]
    rng = random.Random(3)
    pos = [[rng.randint(-5, 100000), rng.randint(0, 44), rng.randint(0, 79)] for _ in range(15)]
    for kw in (dict(positions=pos), dict(positions=pos, pairs=(64, 0, 0), theta=5e5), dict(pairs=(10, 20, 34)),
               dict(wide=True), dict(with_q=False), dict(in_place=True), dict(wide=True, positions=pos)):
        check_append(Case(news, lens, dtype=dtype, pad=2), 8, **kw)


def test_append_many_sequences_and_one_long():
    rng = random.Random(9)
    lens = [rng.randint(1, 40) for _ in range(300)]
    check_append(Case([1] * 300, lens, hk=1, group=2, d=64, pad=12), 2)
    check_append(Case([1500], [1600], hk=2, group=1, page=64), 2)


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "num_pages"])
def test_append_into_holes_and_missing_tokens(bad):
    c = Case([20, 6, 3, 5], [40, 2, 0, 100], columns=4)
    c.b.table[0, 2] = c.n_pages if bad == "num_pages" else bad
    check_append(c, 8)


# ---- together ----------------------------------------------------------------------
def test_prompt_then_tokens_equals_one_causal_pass():
    """Prompts appended and attended in slices, then token by token: every output is the
    causal attention of the whole sequence, from the inputs alone."""
    torch.manual_seed(4)
    hk, hq, d, page = 2, 6, 128, 32
    plan = [[70, 1, 33], [1, 1, 1], [30, 0, 1], [1, 1, 1], [5, 3, 0], [1, 1, 1]]     # new tokens per call
    total = [sum(p[s] for p in plan) for s in range(3)]
    x = [[torch.randn((n, h, d), device=DEV).to(BF16) for h in (hq, hk, hk)] for n in total]
    cols = -(-max(total) // page)
    n_pages = 3 * cols
    kp = torch.full((n_pages, hk, page, d), math.nan, dtype=BF16, device=DEV)
    vp = torch.full_like(kp, math.nan)
    tb = torch.randperm(n_pages, device=DEV).to(torch.int32).reshape(3, cols)
    done, outs = [0, 0, 0], [[], [], []]
    for news in plan:
        rows = [[x[s][a][done[s]:done[s] + news[s]] for s in range(3)] for a in range(3)]
        q, k, v = (torch.cat(r) for r in rows)
        done = [a + n for a, n in zip(done, news)]
        starts = [0, news[0], news[0] + news[1], sum(news)]
        qs = torch.tensor(starts, dtype=torch.int32, device=DEV)
        kl = torch.tensor(done, dtype=torch.int32, device=DEV)
        qr = ff.paged_append(k, v, kp, vp, qs, kl, tb, q=q)
        o = ff.paged_attention(qr, kp, vp, qs, kl, tb, max_new=max(news))
        for s in range(3):
            outs[s].append(o[starts[s]:starts[s + 1]])
    pairs = ref.rope_split(d)
    for s in range(3):
        q, k, v = (ref.f64(t) for t in x[s])
        q, k = (np.stack([ref.rotate(r, [i] * 3, pairs, 10000.0) for i, r in enumerate(t)]) for t in (q, k))
        got = ref.f64(torch.cat(outs[s]))
        for i in range(total[s]):
            for h in range(hq):
                sc = k[:i + 1, h // 3] @ q[i, h] / math.sqrt(d)
                p = np.exp(sc - sc.max())
                want = p @ v[:i + 1, h // 3] / p.sum()
                mean = p @ np.abs(v[:i + 1, h // 3]) / p.sum()
                # Q and K are rounded to bf16 after the rotation: each score moves by at most
                # (2 2^-8 + 2^-16) sum |q k| / sqrt(d), a weight by the exponential of twice that
                e = (2 * ref.U_BF16 + 2.0 ** -16) * np.max(np.abs(k[:i + 1, h // 3]) @ np.abs(q[i, h])) / math.sqrt(d)
                tol = 1.05 * (ref.U_BF16 + math.expm1(2 * e)) * (mean + np.abs(want)) + ref.U_BF16 * np.abs(want) + 1e-4
                assert (np.abs(got[i, h] - want) <= tol).all(), (s, i, h)


def test_block_equals_the_renderer_caches_read_set():
    """A renderer chunk over [anchors | W chunks | itself] by ff_chunk_attention and as a block over
    a paged sequence [anchors | older chunks | W chunks | the chunk]."""
    torch.manual_seed(8)
    heads, d, gh, gw, W, n = 2, 128, 5, 7, 2, 5
    G = gh * gw
    nq = 3 * G
    cache = ff.RendererCache(stages=1, layers=1, ring_chunks=W, frames_per_chunk=3, grid_h=gh, grid_w=gw,
                             heads=heads, head_dim=d, max_anchor_frames=2, device=DEV)
    page, length = 64, 2 * G + n * nq
    cols = -(-length // page)
    kp = torch.full((cols, heads, page, d), math.nan, dtype=BF16, device=DEV)
    vp = torch.full_like(kp, math.nan)
    tb = torch.randperm(cols, device=DEV).to(torch.int32)[None]
    at = 0

    def add(k, v, frames):
        nonlocal at
        at += k.shape[0]
        pos = torch.tensor([[t, y, z] for t in frames for y in range(gh) for z in range(gw)], dtype=torch.int32, device=DEV)
        qs = torch.tensor([0, k.shape[0]], dtype=torch.int32, device=DEV)
        kl = torch.tensor([at], dtype=torch.int32, device=DEV)
        return qs, kl, pos

    ak, av = (torch.randn((2 * G, heads, d), device=DEV).to(BF16) for _ in range(2))
    qs, kl, pos = add(ak, av, [0, 20])
    ff.paged_append(ak, av, kp, vp, qs, kl, tb, positions=pos)
    cache.rope3d(None, ak, [0, 20])
    cache.anchor_set(0, [0, 20], ak, av)
    for c in range(n):
        q, k, v = (torch.randn((nq, heads, d), device=DEV).to(BF16) for _ in range(3))
        frames = [3 * c, 3 * c + 1, 3 * c + 2]
        qs, kl, pos = add(k, v, frames)
        qr = ff.paged_append(k, v, kp, vp, qs, kl, tb, q=q, positions=pos)
        cache.rope3d(q, k, frames)
        assert torch.equal(qr, q)
        mine = ff.paged_attention(qr, kp, vp, qs, kl, tb, block=True, window=W * nq, anchor_tokens=2 * G)
        want = cache.chunk_attention(0, 0, c, q, k, v)
        cache.kv_publish(0, 0, c, k, v)
        # both are within the bf16 bar of the exact result
        assert (mine.float() - want.float()).abs().max() <= 4e-2
        assert (mine.float() - want.float()).norm() <= 1e-2 * want.float().norm()


def test_same_call_same_bits_and_streams():
    c = Case([1, 40, 1], [5000, 900, 70])
    kp, vp, qs, kl, tb = c.on_gpu()
    q = c.q.to(DEV)
    first = ff.paged_attention(q, kp, vp, qs, kl, tb)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for st in side:
        st.wait_stream(torch.cuda.current_stream())
    for i in range(6):
        outs.append(ff.paged_attention(q, kp, vp, qs, kl, tb, stream=side[i % 2]))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)


def test_graph_follows_growing_sequences():
    """Append and attention captured once and replayed while lengths, pages and inputs change on
    the device; eager calls between the replays; a second graph with a workspace of its own."""
    torch.manual_seed(3)
    hk, hq, d, page, cols, S = 2, 8, 128, 16, 40, 5
    n_pages = S * cols
    i32 = dict(dtype=torch.int32, device=DEV)
    kp, vp = (torch.randn((n_pages, hk, page, d), device=DEV).to(BF16) for _ in range(2))
    tb = torch.randperm(n_pages, device=DEV).to(torch.int32).reshape(S, cols).contiguous()
    qs = torch.arange(S + 1, **i32)
    kl = torch.tensor([1, 30, 600, 17, 250], **i32)
    q, k, v = (torch.randn((S + 3, h, d), device=DEV).to(BF16) for h in (hq, hk, hk))
    bytes_ = ff.paged_attention_workspace(q, kp, qs, kl, tb, max_new=1)
    graphs, kept = [], []
    for _ in range(2):
        ws = torch.empty(max(bytes_, 16), dtype=torch.uint8, device=DEV)
        qr, out = torch.zeros_like(q), torch.zeros_like(q)

        def step(ws=ws, qr=qr, out=out):
            ff.paged_append(k, v, kp, vp, qs, kl, tb, q=q, q_out=qr)
            ff.paged_attention(qr, kp, vp, qs, kl, tb, max_new=1, out=out, workspace=ws)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append((g, out))
        kept += [ws, qr]     # a graph does not hold the tensors that it works on
    for it in range(4):
        kl += 1
        q.copy_(torch.randn(q.shape, device=DEV))
        k.copy_(torch.randn(k.shape, device=DEV))
        tb[0] = tb[0].flip(0)
        pools = kp.clone(), vp.clone()
        qe = ff.paged_append(k, v, *pools, qs, kl, tb, q=q)
        want = ff.paged_attention(qe, *pools, qs, kl, tb, max_new=1)
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert torch.equal(out[:S], want[:S])
            assert (out[S:] == 0).all()
        assert torch.equal(kp, pools[0]) and torch.equal(vp, pools[1])
