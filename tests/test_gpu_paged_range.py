"""Values of up to 2^127 in a paged cache, half of the largest finite one: the weighted sums that
are not yet divided pass float32's range, the results do not.  Small ones keep their bits."""
from __future__ import annotations

import pytest
import torch

from paper_2609_32540_amd import ff

from test_gpu_paged import BF16, F32, Case

pytestmark = pytest.mark.gpu

TOP = 2.0 ** 127


def fill(c: Case, keys=None, rising=False):
    """V is 0 but at the given keys of every sequence (all by default): there +-2^127 in turn over the
    columns.  Scores are 0, so that every key weighs the same, or rise by 43 log2 units along the cache."""
    c.q.zero_()
    sign = torch.ones(c.q.shape[2])
    sign[1::2] = -1.0
    top = (TOP * sign).to(c.dtype)
    for s, length in enumerate(c.b.kv_len):
        for j in range(length):
            p, slot = c.b.place(s, j)
            c.v_pages[p, :, slot] = top if keys is None or j in keys else 0.0
            if rising:
                c.k_pages[p, :, slot, 0] = 30.0 * j / length
    if rising:
        c.q[:, :, 0] = 8.0 if c.q.shape[2] == 64 else 8.0 * 2 ** 0.5
    return c


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys", [[0, 48, 80], [5, 3500, 7005]])
def test_keys_of_several_waves_and_parts(dtype, d, keys):
    """One key in a wave's block, in a part."""
    for news in (1, 3):
        c = Case([news], [9001], dtype=dtype, d=d, hk=1, group=7, page=64)
        fill(c, keys).check_attention(heads=[0, 6])


# the keys of one wave's block, of several waves, of several parts, all
KEYS = [range(4), range(0, 256, 16), range(5, 9000, 1000), None]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys", KEYS)
def test_few_rows(dtype, d, keys):
    """A short cache (waves joined) and a long one (parts joined)."""
    for news, length in (([1], 300), ([1], 9001), ([3], 9001)):
        c = Case(news, [length], dtype=dtype, d=d, hk=1, group=7, page=64)
        fill(c, keys).check_attention(heads=[0, 6])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("news,length", [(1, 300), (20, 300), (1, 9001)])
def test_few_rows_under_rising_scores(dtype, news, length):
    fill(Case([news], [length], dtype=dtype, d=64, hk=1, group=2, page=64), rising=True).check_attention(rows=[0, news - 1])


@pytest.mark.parametrize("news,length,hk,form", [(700, 1000, 64, (0, 0, 256, 0)), (256, 24000, 4, (0, 0, 256, 1))])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys,rising", [(range(4), False), (range(5, 9000, 100), False), (None, False), (None, True)])
def test_prompts(news, length, hk, form, d, keys, rising):
    """The 256-row kernel, its keys in one part and in several; causal, with a window (no fast pass), and
    as one block."""
    c = fill(Case([news], [length], d=d, hk=hk, group=1, page=64), keys, rising)
    for kw in (dict(), dict(window=length // 2), dict(block=True)):
        c.check_attention(rows=[0, 100, news - 1], heads=[0, hk - 1], min_new=news, form=form, **kw)


@pytest.mark.parametrize("dtype,news,length,hk,group", [
    (BF16, 1, 9001, 1, 4), (F32, 1, 9001, 1, 4), (BF16, 5, 300, 2, 3), (F32, 40, 300, 2, 3), (BF16, 700, 1000, 64, 1),
    (BF16, 256, 24000, 4, 1)])
def test_small_values(dtype, news, length, hk, group):
    """V of 2^-118: the result is that of V, scaled.  Products end at steps of 2^-149.  Where a reference is
    lifted, by at most 16, a weight is above 2^-16 times what it is without, and these scores (standard
    normal) keep the sum of n weights above n / 2^6: n half steps over that sum are 2^-128, 2^-10 of V's
    unit.  The rest is a rounding of either side."""
    c = Case([news], [length], dtype=dtype, d=64, hk=hk, group=group, page=64)
    kp, vp, qs, kl, tb = c.on_gpu()
    q = c.q.to("cuda")
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -22
    for window in (-1, length):
        for lse in (None, torch.empty(q.shape[:2], device="cuda")):
            want = ff.paged_attention(q, kp, vp, qs, kl, tb, window=window, lse=lse, min_new=news).double()
            got = ff.paged_attention(q, kp, vp * 2.0 ** -118, qs, kl, tb, window=window, lse=lse, min_new=news).double()
            assert ((got * 2.0 ** 118 - want).abs() <= 2 * u * want.abs() + 2.0 ** -10).all()
