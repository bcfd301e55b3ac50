"""The paged cache's kernels in each of their forms: workgroups of two waves, float32 prompts in parts,
appends of two rows per block, and the exactness of the bf16 kernel of few rows."""
from __future__ import annotations

import math
import random

import numpy as np
import pytest
import torch

from paper_2609_32540_amd import ff

import paged_ref as ref
from test_gpu_paged import BF16, DEV, F32, Case, check_append

gpu = pytest.mark.gpu


def forms():
    """Of the thread's last call: rows of a tile of few rows, whether its keys could be cut, the same of
    many rows; the waves of a workgroup of few rows, whether its keys are read past the caches."""
    return tuple(ff.lib().ff_internal_last_paged(i) for i in range(6))


# ---- workgroups of two waves -------------------------------------------------------
@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,group,hint,form", [
    (1, 4, 1, (16, 0, 0, 0, 2, 1)), (3, 7, 3, (32, 0, 0, 0, 2, 1)), (3, 7, 0, (32, 0, 0, 0, 2, 0))])
def test_short_caches_in_many_workgroups(d, new, group, hint, form):
    """300 sequences of up to 500 keys, two kv heads: more than two workgroups per compute unit."""
    rng = random.Random(d + new)
    lens = [rng.randint(0, 500) for _ in range(300)]
    lens[:6] = [500, 0, 1, 32, 33, 64]
    news = [min(n, rng.randint(0, new)) for n in lens]
    c = Case(news, lens, d=d, hk=2, group=group)
    some = sorted(set(list(range(20)) + [rng.randrange(c.rows) for _ in range(60)] + [c.rows - 1]))
    for kw in (dict(), dict(block=True, window=70, anchors=20)):
        c.check_attention(rows=some, heads=[0, group, 2 * group - 1], max_new=hint, **kw)
        assert forms() == form


# ---- float32 -----------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news,lens,cut", [([90, 200], [5000, 3100], 1), ([700, 129, 1, 64], [700, 400, 350, 77], 0)])
def test_float32_prompts(d, news, lens, cut):
    c = Case(news, lens, dtype=F32, d=d, hk=1, group=3, page=64)
    for kw in (dict(), dict(block=True), dict(window=300, anchors=70)):
        c.check_attention(rows=[0, 31, 32, 63, 89, 90, 200, sum(news) - 1], **kw)
        assert forms() == (32, cut, 0, 0, 4, 0)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,group,form", [(1, 2, (16, 1, 0, 0, 4, 1)), (4, 5, (32, 1, 0, 0, 4, 1))])
def test_float32_few_tokens(d, new, group, form):
    c = Case([new] * 3, [3000, 40, 1500], dtype=F32, d=d, hk=2, group=group)
    c.check_attention(max_new=new)
    assert forms() == form


# ---- batches that the forms share --------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_long_caches_of_more_sequences_than_lanes(dtype, d):
    """130 sequences, some of them cut into parts."""
    rng = random.Random(d)
    lens = [rng.choice([0, 1, 90, 1500, 3100]) for _ in range(130)]
    c = Case([min(n, 1) for n in lens], lens, dtype=dtype, d=d, hk=1, group=2)
    c.check_attention(max_new=1)
    assert forms()[:2] == (16, 1)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_of_more_sequences_than_lanes(d):
    rng = random.Random(d)
    news = [rng.choice([0, 33, 64, 150]) for _ in range(100)]
    lens = [n + rng.choice([0, 7, 200, 1000]) for n in news]
    c = Case(news, lens, d=d, hk=16, group=4)
    rows = sorted(rng.sample(range(c.rows), 40)) + [c.rows - 1]
    for kw in (dict(), dict(window=100, anchors=20), dict(block=True)):
        c.check_attention(rows=rows, heads=[0, 63], min_new=33, max_new=150, **kw)
        assert forms()[:4] == (0, 0, 256, 0)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_both_kernels_with_their_keys_in_parts(d):
    """A slice of a prompt beside single tokens, long caches, few heads: both kernels leave partial
    results in one workspace."""
    c = Case([1000, 1, 1, 7], [16000, 9000, 300, 5000], d=d, hk=4, group=1, page=64)
    for kw in (dict(), dict(block=True), dict(window=4000, anchors=500)):
        c.check_attention(rows=[0, 255, 256, 999, 1000, 1001, 1002, 1008], heads=[0, 3], **kw)
        assert forms()[:4] == (32, 1, 256, 1)


@gpu
@pytest.mark.parametrize("dtype,news,lens,hk,kw", [
    (BF16, [1], [9001], 2, dict(max_new=1)), (BF16, [1000, 1, 7], [16000, 9000, 5000], 4, {}),
    (BF16, [1000], [16000], 4, dict(min_new=1000)), (F32, [1, 4], [5000, 3000], 2, {}), (F32, [200], [5000], 1, {})])
def test_workspace_is_kept_to_and_not_read_before_it_is_written(dtype, news, lens, hk, kw):
    c = Case(news, lens, dtype=dtype, d=64, hk=hk, group=1, page=64)
    kp, vp, qs, kl, tb = c.on_gpu()
    q = c.q.to(DEV)
    n = ff.paged_attention_workspace(q, kp, qs, kl, tb, **kw)
    assert n > 0
    want = ff.paged_attention(q, kp, vp, qs, kl, tb, **kw)
    for fill in (0xFF, 0x00):      # (0xFF: NaN)
        wide = torch.full((4096 + n + 4096,), fill, dtype=torch.uint8, device=DEV)
        got = ff.paged_attention(q, kp, vp, qs, kl, tb, workspace=wide[4096:4096 + n], **kw)
        assert torch.equal(got, want)
        assert (wide[:4096] == fill).all() and (wide[4096 + n:] == fill).all()


# ---- appends -----------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,pad", [(1501, 0), (1500, 1), (1499, 3)])
def test_append_two_rows_per_block(dtype, d, rows, pad):
    """An odd count leaves a block of one row; sequences that begin and end inside a block."""
    check_append(Case([3, rows - 4, 1], [3, rows + 96, 70], dtype=dtype, d=d, hk=1, group=2, page=64, pad=pad), 2)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_text_turns_one_axis_by_the_index(dtype, d):
    """No positions and all pairs on one axis: the rotation of a text model."""
    for theta in (1e4, 5e5):
        check_append(Case([1, 0, 9, 40], [700, 5, 9, 3000], dtype=dtype, d=d, hk=2, group=2), 4, pairs=(d // 2, 0, 0), theta=theta)


# ---- exactness ---------------------------------------------------------------------
def bf16(x):
    """Nearest bf16 values of float64 ones."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(BF16).double().numpy()


def causal_row(c: Case, s: int, i: int, row: int, head: int):
    """(weights, V rows, bound) of a query: the exact row is weights @ V / sum, and the bound that
    of paged_ref.attention with u_p = 2^-17, a weight as two bf16 (its value rounded and what that leaves
    rounded again), 32 float32 steps for the joins of waves and parts, and half a step of the result
    itself in place of the relative one."""
    hk, d = c.k_pages.shape[1], c.q.shape[2]
    h = head // (c.q.shape[1] // hk)
    at = [c.b.place(s, j) for j in range(i + 1)]
    pg, sl = torch.tensor([x[0] for x in at]), torch.tensor([x[1] for x in at])
    k, v, q = ref.f64(c.k_pages[pg, h, sl]), ref.f64(c.v_pages[pg, h, sl]), ref.f64(c.q[row, head])
    x = k @ q / math.sqrt(d)
    p = np.exp(x - x.max())
    out, mean = p @ v / p.sum(), p @ np.abs(v) / p.sum()
    e = 2 * (d + 8) * ref.U_F32 * float(np.max(np.abs(k) @ np.abs(q))) / math.sqrt(d) + (40 + len(p)) * ref.U_F32
    off = 1.05 * (2.0 ** -17 + e) * (mean + np.abs(out))
    half = 2.0 ** (np.floor(np.log2(np.abs(out) + off)) - 8)
    return p, v, out, off + half + 1e-30


EXACT = [([1, 1], [700, 90], 0), ([1], [9001], 0), ([5, 17], [300, 2000], 0), ([200], [350], 0), ([1, 3], [700, 500], 1)]


def exact_case(news, lens, top, d):
    c = Case(news, lens, d=d, hk=1, group=3, seed=d)
    if top:                 # values whose sums pass float32's range: the second run of a wave
        c.v_pages *= 2.0 ** 125
    return c


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news,lens,top", EXACT)
def test_few_rows_are_as_exact_as_their_rounding(news, lens, top, d):
    c = exact_case(news, lens, top, d)
    kp, vp, qs, kl, tb = c.on_gpu()
    got = ref.f64(ff.paged_attention(c.q.to(DEV), kp, vp, qs, kl, tb))
    assert forms()[0] in (16, 32) and forms()[2] == 0
    for row, s, i in c.b.tokens(c.rows):
        if row % 7 in (0, 3):
            for head in (0, 2):
                _, _, out, tol = causal_row(c, s, i, row, head)
                assert (np.abs(got[row, head] - out) <= tol).all(), (row, head)


@pytest.mark.parametrize("news,lens,top", [x for x in EXACT if max(x[1]) <= 2000])
def test_the_bound_tells_one_rounding_from_two(news, lens, top):
    """On the CPU: weights of one bf16 are outside the bound, weights of two inside.  (Over 9001 keys the
    bound of the float32 sums is wider than either.)"""
    c = exact_case(news, lens, top, 64)
    once = twice = 0
    for row, s, i in c.b.tokens(c.rows):
        if row % 7 in (0, 3):
            p, v, out, tol = causal_row(c, s, i, row, 0)
            hi = bf16(p)
            once += (np.abs(bf16(hi @ v / p.sum()) - out) > tol).sum()
            twice += (np.abs(bf16((hi + bf16(p - hi)) @ v / p.sum()) - out) > tol).sum()
    assert twice == 0 and once > 0
