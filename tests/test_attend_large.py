"""Calls of more query rows, and of more blocks, than 2^24."""
import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_many_query_rows(dtype):
    """One token's query, read by all tokens (its stride along them is 0): every output is that token's."""
    N, D, T = (1 << 24) + 5, 8, 40
    q, K, V = rand(1, 1, 1, D, dtype=dtype, seed=1), rand(1, 1, T, D, dtype=dtype, seed=2), rand(1, 1, T, D, dtype=dtype, seed=3)
    print("[gpu-test] many query rows", dtype, flush=True)
    got = lagkv.attend(q.expand(1, 1, N, D), K, V, want_lse=True)
    assert bool((got.out == got.out[:, :, :1]).all()) and bool((got.lse == got.lse[:, :, :1]).all())
    A.check(lagkv.Attended(got.out[:, :, :1].clone(), got.lse[:, :, :1].clone()), A.attend(q, K, V))
    # the last tokens of a causal prompt see all before them: here with rows that all are one
    if dtype == torch.bfloat16:
        N = 1 << 13
        heads = 1 << 11
        got = lagkv.attend(q.expand(1, heads, N, D), K[:, :, :0], V[:, :, :0], K[:, :, :1].expand(1, 1, N, D), V[:, :, :1].expand(1, 1, N, D))
        assert bool((got.out == V[:, :, :1]).all())


def test_many_blocks():
    """8192 streams of 2048 blocks; the same bounds and queries in all of them (strides of 0)."""
    B, H, G, D, nb, k = 1024, 8, 4, 64, 2048, 64
    lo = rand(1, 1, nb, D, dtype=torch.bfloat16, seed=4)
    hi = lo + rand(1, 1, nb, D, dtype=torch.bfloat16, seed=5).abs()
    q = rand(1, 1, 1, D, dtype=torch.bfloat16, seed=6)
    print("[gpu-test] many blocks", flush=True)
    got = lagkv.select_blocks(q.expand(B, H * G, 1, D), lo.expand(B, H, nb, D), hi.expand(B, H, nb, D), nb * 64, 64, k, 1, 4)
    assert bool((got == got[:1, :1]).all())
    assert torch.equal(got[:1, :1].cpu(), A.select(q.expand(1, G, 1, D), lo, hi, nb * 64, 64, k, 1, 4))
