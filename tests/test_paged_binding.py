"""What the binding of the paged cache refuses before the library sees it: integers past 32 bits and
arguments that are not tensors."""
import pytest
import torch

from paper_2609_32540_amd import ff

I32 = dict(dtype=torch.int32)
BF16 = torch.bfloat16


def tensors(dev):
    pool = torch.zeros((4, 2, 16, 128), dtype=BF16, device=dev)
    batch = torch.tensor([0, 1], device=dev, **I32), torch.tensor([5], device=dev, **I32), torch.zeros((1, 2), device=dev, **I32)
    return torch.zeros((1, 8, 128), dtype=BF16, device=dev), torch.zeros((1, 2, 128), dtype=BF16, device=dev), pool, batch


@pytest.mark.parametrize("pairs", [(2 ** 32 + 22, 21, 21), (64, 0, 2 ** 32), (64 - 2 ** 32, 0, 0)])
def test_rope_pairs_past_32_bits(pairs):
    _, k, pool, batch = tensors("cpu")
    with pytest.raises(ValueError, match="32 bits"):
        ff.paged_append(k, k, pool, pool, *batch, rope_pairs=pairs)


@pytest.mark.parametrize("kw", [dict(q_out=[1]), dict(positions=[[0, 0, 0]]), dict(positions=5)])
def test_append_arguments_that_are_no_tensors(kw):
    q, k, pool, batch = tensors("cpu")
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        ff.paged_append(k, k, pool, pool, *batch, q=q, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("hint", [dict(min_new=-2 ** 32), dict(max_new=1 - 2 ** 32), dict(min_new=1, max_new=2 ** 31)])
def test_hints_past_32_bits(hint):
    q, _, pool, batch = tensors("cuda")
    with pytest.raises(ValueError, match="32 bits"):
        ff.paged_attention(q, pool, pool, *batch, **hint)
    with pytest.raises(ValueError, match="32 bits"):
        ff.paged_attention_workspace(q, pool, *batch, **hint)


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(out=[1]), dict(lse=3.0), dict(workspace=b"1234")])
def test_attention_arguments_that_are_no_tensors(kw):
    q, _, pool, batch = tensors("cuda")
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        ff.paged_attention(q, pool, pool, *batch, **kw)
