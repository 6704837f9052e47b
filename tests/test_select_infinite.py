"""The selection of blocks whose bounds are infinite (an overflowed key is enough): by the score as it is defined, whatever the number of
channels and of tokens; behind all others where that is not finite."""
import math

import pytest
import torch

from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def scores(q, lo, hi, G):
    """[B,H,N,nb] in 64 bits: sum over the query heads and channels of max(q lo, q hi)."""
    B, HG, N, D = q.shape
    x = q.double().view(B, HG // G, G, N, 1, D)
    return torch.maximum(x * lo.double()[:, :, None, None], x * hi.double()[:, :, None, None]).sum((2, 5))


def select(s, k, first, last, held):
    out = torch.full((*s.shape[:3], k), -1, dtype=torch.int32)
    for b in range(s.shape[0]):
        nb = held[b]
        for h in range(s.shape[1]):
            for n in range(s.shape[2]):
                v = s[b, h, n].tolist()
                key = lambda j: (not (j < first or j >= nb - last), -v[j] if math.isfinite(v[j]) else math.inf, j)
                got = sorted(sorted(range(nb), key=key)[:k])
                out[b, h, n, :len(got)] = torch.tensor(got, dtype=torch.int32)
    return out


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [8, 13, 41, 64, 72, 80, 100, 128, 200, 256])
@pytest.mark.parametrize("N", [1, 3, 4, 17])
def test_infinite_bounds(dtype, D, N):
    print("[gpu-test] infinite bounds", dtype, D, N, flush=True)
    B, H, G, block, nb, k = 2, 2, 3, 16, 150, 40
    g = torch.Generator().manual_seed(D + N)
    lo = torch.randn(B, H, nb, D, generator=g).to(dtype)
    hi = (lo.float() + torch.rand(B, H, nb, D, generator=g)).to(dtype)
    q = torch.randn(B, H * G, N, D, generator=g).to(dtype)
    q[:, :, :, 0] = -q[:, :, :, 0].abs() - 0.25            # below 0 in every head: hi = inf leaves the score finite
    q[:, :, :, D - 1] = q[:, :, :, D - 1].abs() + 0.25     # above 0: lo = -inf does
    q[:, ::4, :, 5] = 0.0                                  # 0 in some heads
    q[:, :, :, 6] = 0.0                                    # and in all
    for j in range(nb):
        kind = j % 12
        if kind == 0:
            hi[:, :, j, 0] = math.inf
        elif kind == 1:
            lo[:, :, j, D - 1] = -math.inf
        elif kind == 2:
            hi[:, :, j, 0], lo[:, :, j, D - 1] = math.inf, -math.inf
        elif kind == 3 and j % 24 == 3:
            lo[:, :, j, 0] = -math.inf                     # +inf
        elif kind == 4 and j % 24 == 4:
            lo[:, :, j, 0] = hi[:, :, j, 0] = math.inf     # -inf
        elif kind == 5:
            hi[:, :, j, 5] = math.inf                      # NaN where q is 0 in a head
        elif kind == 6 and j % 24 == 6:
            lo[:, :, j, 3], hi[:, :, j, 3] = math.inf, -math.inf
        elif kind == 7 and j % 24 == 7:
            hi[:, :, j, 2] = math.nan
        elif kind == 8:
            lo[:, :, j, 5] = -math.inf
        elif kind == 9 and j % 24 == 9:
            hi[:, :, j, 6] = math.inf
        elif kind == 10:
            hi[:, :, j, 0], lo[:, :, j, 0] = -0.5, math.inf  # (out of order)
    T = nb * block - 5
    lengths = torch.tensor([T, 100 * block + 1], dtype=torch.int32)
    held = [nb, 101]
    lo[1, :, 101:], hi[1, :, 101:] = math.inf, -math.inf    # (as block_bounds leaves blocks without rows)
    s = scores(q, lo, hi, G)
    assert bool(torch.isfinite(s[:, :, :, 0:101:12]).all()) and bool((s[:, :, :, 3:101:24] == math.inf).all())
    lo, hi, q = lo.to(DEV), hi.to(DEV), q.to(DEV)
    for first, last in ((0, 0), (1, 2)):
        got = lagkv.select_blocks(q, lo, hi, T, block, k, first, last, lengths.to(DEV)).cpu()
        assert torch.equal(got, select(s, k, first, last, held)), (first, last)
    every = lagkv.select_blocks(q, lo, hi, T, block, 99, 0, 0, lengths.to(DEV)).cpu()
    assert torch.equal(every, select(s, 99, 0, 0, held))


@pytest.mark.parametrize("N", [1, 5])
def test_an_overflowed_key(N):
    """An fp16 key of -inf: attention over its block is finite, and the selection takes the block for what its score is."""
    D, T = 80, 64 * 16
    g = torch.Generator().manual_seed(3)
    K = torch.randn(1, 1, T, D, generator=g).half()
    q = torch.randn(1, 2, N, D, generator=g).half()
    q[..., 2] = q[..., 2].abs() + 0.25
    K[0, 0, 333, 2] = -math.inf
    K[0, 0, 334:336] += 3 * q[0, :].sum((0, 1)).sign()
    K, q = K.to(DEV), q.to(DEV)
    lo, hi = lagkv.block_bounds(K, 16)
    blocks = lagkv.select_blocks(q, lo, hi, T, 16, 8)
    s = scores(q.cpu(), lo.cpu(), hi.cpu(), 2)
    assert torch.equal(blocks.cpu(), select(s, 8, 0, 0, [64]))
    assert 20 in blocks[0, 0, 0].tolist()                  # (row 333's)
    got = lagkv.attend_blocks(q, K, torch.randn(1, 1, T, D, generator=g).half().to(DEV), blocks, 16, want_lse=True)
    assert bool(torch.isfinite(got.out).all()) and bool(torch.isfinite(got.lse).all())
