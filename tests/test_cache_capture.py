"""A captured step that goes through a cache's layers, and what its calls read."""
import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

DEV = "cuda:0"


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def test_whose_stream_is_captured(monkeypatch):
    """A cache on a device that is not the current one: it is its own device's stream that counts."""
    now = [0]

    class Guard:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, now[0] = now[0], self.device.index

        def __exit__(self, *a):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now[0] == 1)
    seen = []

    class Keys:
        device, is_cuda, shape = torch.device("cuda", 1), True, (1, 1, 64, 8)

        def __getitem__(self, at):
            return self

    cache = lagkv.Cache(1, 1, 8, 64, 2, 16, 0.5, device="cpu")
    cache.K, cache.c.n_static = Keys(), 40
    monkeypatch.setattr(lagkv, "block_bounds", lambda K, block: seen.append(K) or ("lo", "hi"))
    assert cache.block_bounds(16) == ("lo", "hi") and len(seen) == 1 and cache._bounds == {} and now == [0]


@pytest.mark.gpu
def test_a_captured_step_reads_every_layer_once(monkeypatch):
    layers, B, H, G, D, T, block, k = 4, 2, 2, 4, 64, 600, 16, 5
    cache = lagkv.Cache(layers * B, H, D, 700, 4, 32, 0.5)
    x = rand(layers * B, H, T, D, dtype=torch.bfloat16, seed=8)
    cache.K.zero_()
    cache.V.zero_()
    cache.c.n_static, cache.c.n_seen = T, T
    q = rand(layers, B, H * G, 1, D, dtype=torch.bfloat16, seed=9)
    of = [slice(i * B, (i + 1) * B) for i in range(layers)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        lagkv.select_blocks(q[0], *lagkv.block_bounds(x[:B], block), T, block, k)
    torch.cuda.synchronize()
    read, whole = [], lagkv.block_bounds
    monkeypatch.setattr(lagkv, "block_bounds", lambda K, *a, **kw: read.append(tuple(K.shape)) or whole(K, *a, **kw))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        picked = [cache.select_blocks(q[i], block, k, 1, 1, batch=of[i]) for i in range(layers)]
        some = [cache.attend_blocks(q[i], picked[i], block, batch=of[i]).out for i in range(layers)]
    monkeypatch.undo()
    assert read == [(B, H, T, D)] * layers and cache._bounds == {}
    for turn in range(3):
        rows = x * (turn - 1.5)
        cache.K[:, :, :T].copy_(rows)
        cache.V[:, :, :T].copy_(rows.flip(2))
        graph.replay()
        torch.cuda.synchronize()
        for i in range(layers):
            lo, hi = A.bounds(rows[of[i]], block)
            assert torch.equal(picked[i].cpu(), A.select(q[i], lo, hi, T, block, k, 1, 1)), (turn, i)
            A.check(lagkv.Attended(some[i], None), A.attend(q[i], rows[of[i]], rows.flip(2)[of[i]], blocks=picked[i].cpu(), block=block))
        cache.changed_from(0)
        lo, hi = cache.block_bounds(block)                  # eager work in between
        wl, wh = A.bounds(rows, block)
        assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
        cache._bounds.clear()
