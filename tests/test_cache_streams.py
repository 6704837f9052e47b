"""The bounds that a cache keeps, read on another stream than the one they were made on."""
import pytest
import torch

from paper_2504_04704_amd import lagkv

DEV = "cuda:0"


@pytest.mark.gpu
def test_kept_bounds_outlive_the_cache_while_another_stream_reads_them():
    B, H, D, T, block = 2, 2, 128, 4000, 16
    x = torch.randn(B, H, T, D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    q = torch.randn(B, 2 * H, 1, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    want = lagkv.select_blocks(q, *lagkv.block_bounds(x, block), T, block, 20)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    busy = torch.zeros(4096, 4096, device=DEV)
    torch.mm(busy, busy)
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        cache = lagkv.Cache(B, H, D, 4096, 4, 128, 0.25)
        cache.K[:, :, :T].copy_(x)
        cache.c.n_static, cache.c.n_seen = T, T
        lo, hi = cache.block_bounds(block)
        mine = {lo.data_ptr(), hi.data_ptr()}
        shape = cache._bounds[block][0].shape
    del lo, hi
    with torch.cuda.stream(b):
        b.wait_stream(a)
        for _ in range(40):
            busy = torch.mm(busy, busy)
        got = cache.select_blocks(q, block, 20)
        done = torch.cuda.Event()
        done.record()
    del cache
    with torch.cuda.stream(a):
        new = [torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    still = not done.query()
    assert still and not mine & {t.data_ptr() for t in new}
    torch.cuda.synchronize()
    assert torch.equal(got, want)
