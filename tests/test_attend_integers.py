"""Integers that a 32-bit field of the parameters does not hold are refused, before any device work: what is left of 2**32 + 16 is a
block of 16 rows, whose bounds are more than the buffers for one of 2**32 + 16 rows take."""
import pytest
import torch

from paper_2504_04704_amd import lagkv

FAR = [2 ** 32 + 16, 2 ** 31, -2 ** 32 + 16, 2 ** 64 + 32]


def refused(f, *a, **kw):
    with pytest.raises(lagkv.LagKVError) as e:
        f(*a, **kw)
    assert e.value.status == lagkv.EINVAL


@pytest.mark.parametrize("n", FAR)
def test_blocks_and_counts(n):
    q, K, lo = torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 50, 64), torch.zeros(1, 2, 4, 64)
    blocks = torch.zeros(1, 2, 1, 3, dtype=torch.int32)
    refused(lagkv.block_bounds, K, n)
    refused(lagkv.attend_blocks, q, K, K, blocks, n)
    refused(lagkv.select_blocks, q, lo, lo, 50, n, 2)
    refused(lagkv.select_blocks, q, lo, lo, 50, 16, n)
    refused(lagkv.select_blocks, q, lo, lo, 50, 16, 2, n)
    refused(lagkv.select_blocks, q, lo, lo, 50, 16, 2, 0, n)
    cache = lagkv.Cache(1, 1, 64, 40, 2, 16, 0.5, device="cpu")
    cache.c.n_tail = 30
    refused(lagkv.block_bounds, cache.K, n)


def test_sizes():
    """(Tensors of one row, repeated.)"""
    far = 2 ** 32 + 1
    q, K = torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 1, 64)
    refused(lagkv.attend, q.expand(1, 4, far, 64), K, K)
    refused(lagkv.attend, q[:, :1].expand(far, 1, 1, 64), K[:, :1].expand(far, 1, 1, 64), K[:, :1].expand(far, 1, 1, 64))
    refused(lagkv.block_bounds, K.expand(1, 2, far, 64), 16)
    refused(lagkv.select_blocks, q, K.expand(1, 2, far, 64), K.expand(1, 2, far, 64), 16 * far, 16, 2)
    refused(lagkv.attend_blocks, q, K, K, torch.zeros(1, 2, 1, 1, dtype=torch.int32).expand(1, 2, 1, far), 16)
