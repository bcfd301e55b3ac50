"""Values of up to 2^127 in a paged cache, half of the largest finite one: the weighted sums that
are not yet divided pass float32's range, the results do not."""
from __future__ import annotations

import pytest
import torch

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
