"""A cache in use: compressed in prefill, read by every layer of a step (all rows, or blocks that are selected), the rows of the
accepted path of a drafted tree appended and compressed, its bounds kept up to date meanwhile."""
import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

DEV = "cuda:0"


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float16, 80), (torch.float32, 64)], ids=["bf16", "f16", "f32"])
def test_steps_of_a_model(dtype, D):
    layers, B, H, G, S, L, r, block, N = 2, 2, 2, 4, 4, 32, 0.25, 16, 6
    cache = lagkv.Cache(layers * B, H, D, 400, S, L, r, dtype=dtype)
    K, V = rand(layers * B, H, 500, D, dtype=dtype, seed=1), rand(layers * B, H, 500, D, dtype=dtype, seed=2)
    cache.block_bounds(block)                                  # (of nothing)
    cache.prefill_chunked(K, V)
    parents = torch.tensor([-1, 0, 0, 1, 3, 2], dtype=torch.int32, device=DEV)
    path = [0, 1, 3, 4]                                        # what the model accepts of every tree
    rounds = 0
    for step in range(24):
        Kn, Vn = rand(layers * B, H, N, D, dtype=dtype, seed=100 + step), rand(layers * B, H, N, D, dtype=dtype, seed=200 + step)
        for layer in range(layers):
            at = slice(layer * B, (layer + 1) * B)
            q = rand(B, N, H * G, D, dtype=dtype, seed=300 + step + 50 * layer).transpose(1, 2)
            k, v, _ = cache.view()
            every = cache.attend(q, Kn[at], Vn[at], parents, batch=at, want_lse=True)
            blocks = cache.select_blocks(q, block, 3, 1, 1, batch=at)
            some = cache.attend_blocks(q, blocks, block, Kn[at], Vn[at], parents, batch=at, want_lse=True)
            if step % 6 == 0:
                A.check(every, A.attend(q, k[at], v[at], Kn[at], Vn[at], parents), f"step {step}")
                A.check(some, A.attend(q, k[at], v[at], Kn[at], Vn[at], parents, blocks=blocks.cpu(), block=block), f"step {step}")
        lo, hi = cache.block_bounds(block)
        wl, wh = A.bounds(cache.view()[0], block)
        assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh), step
        static = cache.n_static
        cache.append_and_compress(Kn[:, :, path], Vn[:, :, path])
        rounds += cache.n_static != static
    assert rounds >= 2
    # a second size of block, and rows written past the object's calls
    cache.block_bounds(32)
    cache.K[:, :, 7] = 3.0
    cache.changed_from(7)
    for size in (16, 32):
        lo, hi = cache.block_bounds(size)
        wl, wh = A.bounds(cache.view()[0], size)
        assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
    out = lagkv.compress(K, V, S, L, r)
    again = lagkv.Cache.from_compressed(out, 500, 400, S, L, r)
    lo, hi = again.block_bounds(block)
    assert torch.equal(lo.cpu(), A.bounds(out.K, block)[0])


@pytest.mark.gpu
def test_bounds_on_two_streams():
    """The stream of a call that finds the bounds kept does not run ahead of the one that they are made on."""
    cache = lagkv.Cache(2, 2, 128, 4096, 4, 128, 0.25)
    x = rand(2, 2, 4000, 128, dtype=torch.bfloat16, seed=8)
    cache.K[:, :, :4000].copy_(x)
    cache.c.n_static, cache.c.n_seen = 4000, 4000
    q = rand(2, 4, 1, 128, dtype=torch.bfloat16, seed=9)
    want = lagkv.select_blocks(q, *lagkv.block_bounds(x, 16), 4000, 16, 20)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    busy = torch.zeros(4096, 4096, device=DEV)
    torch.mm(busy, busy)
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        for _ in range(20):
            busy = torch.mm(busy, busy)
        first = cache.select_blocks(q, 16, 20)
    with torch.cuda.stream(b):
        second = cache.select_blocks(q, 16, 20)
    torch.cuda.synchronize()
    assert torch.equal(first, want) and torch.equal(second, want)


@pytest.mark.gpu
def test_bounds_in_a_captured_step():
    """A captured step works the bounds out in every replay, and leaves those of the steps outside it alone."""
    cache = lagkv.Cache(1, 2, 64, 700, 4, 32, 0.5)
    x = rand(1, 2, 600, 64, dtype=torch.bfloat16, seed=8)
    cache.K.zero_()
    cache.V.zero_()
    cache.c.n_static, cache.c.n_seen = 600, 600
    q = rand(1, 4, 1, 64, dtype=torch.bfloat16, seed=9)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        lagkv.select_blocks(q, *lagkv.block_bounds(x, 16), 600, 16, 5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        picked = cache.select_blocks(q, 16, 5)
    for turn in range(3):
        rows = x * (turn - 1.5)
        cache.K[:, :, :600].copy_(rows)
        cache.changed_from(0)
        want = lagkv.select_blocks(q, *lagkv.block_bounds(rows, 16), 600, 16, 5)
        assert torch.equal(cache.select_blocks(q, 16, 5), want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(picked, want), turn
        lo, hi = cache.block_bounds(16)
        wl, wh = A.bounds(rows, 16)
        assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)


@pytest.mark.gpu
def test_a_refused_append_leaves_the_bounds_right():
    cache = lagkv.Cache(1, 1, 64, 40, 2, 16, 0.5)
    x = rand(1, 1, 30, 64, dtype=torch.bfloat16, seed=5)
    cache.append_and_compress(x, x)
    lo, hi = cache.block_bounds(16)
    with pytest.raises(lagkv.LagKVError) as e:
        cache.append_and_compress(x, x)                        # no room
    assert e.value.status == lagkv.ECAPACITY
    lo, hi = cache.block_bounds(16)
    wl, wh = A.bounds(cache.view()[0], 16)
    assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
    cache.append_and_compress(x[:, :, :3], x[:, :, :3])
    wl, _ = A.bounds(cache.view()[0], 16)
    assert torch.equal(cache.block_bounds(16)[0].cpu(), wl)


def test_a_bad_block_is_refused_before_anything_is_kept():
    cache = lagkv.Cache(1, 1, 64, 40, 2, 16, 0.5, device="cpu")
    for block in (0, -16):
        with pytest.raises(lagkv.LagKVError):
            cache.block_bounds(block)
    assert cache._bounds == {}
