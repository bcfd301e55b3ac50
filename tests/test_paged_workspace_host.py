"""Workspace of the paged attention where the keys are cut into parts, without a GPU: it stays a
small part of what the call itself moves, whatever the number of rows and the table's width."""
import ctypes

import pytest

from paper_2609_32540_amd import ff

DEV = 0x7f0000000000     # aligned; never dereferenced here


def workspace(dtype, q_heads, kv_heads, d, tokens, seqs, keys, page=16, **hints):
    cols = -(-keys // page)
    return ff.lib().ff_paged_attention_workspace(ctypes.byref(ff.PagedDesc(
        1 << 20, page, q_heads, kv_heads, d, dtype, seqs, tokens, cols, hints.get("min_new", 0),
        hints.get("max_new", 0), 0, cols, DEV, DEV, DEV)))


@pytest.mark.parametrize("q_heads,kv_heads,tokens,seqs,keys", [
    (64, 8, 8997, 5, 32768 * 16), (96, 12, 4961, 1, 16384 * 16), (64, 8, 33051, 1, 131072 * 16),
    (32, 8, 5000, 1, 5000), (8, 8, 100000, 40, 4096), (64, 64, 700, 1, 1 << 20), (3, 3, 2184, 1, 8736)])
@pytest.mark.parametrize("d", [64, 128])
def test_float32_prompts(q_heads, kv_heads, tokens, seqs, keys, d):
    """Partial results of 32 rows x (d + 2) floats: at most 16 for each of 256 compute units."""
    assert workspace(ff.FF_DT_F32, q_heads, kv_heads, d, tokens, seqs, keys) <= 16 * 256 * 32 * (d + 2) * 4


def test_float32_prompts_of_few_tiles_are_still_cut():
    """207 tiles over 8736 keys leave a fifth of the compute units idle: six parts each."""
    assert workspace(ff.FF_DT_F32, 3, 3, 128, 2184, 1, 8736, page=64) >= 2 * 207 * 32 * 130 * 4
