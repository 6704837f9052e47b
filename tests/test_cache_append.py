"""Appending to a cache whose bounds are kept."""
import pytest
import torch

from paper_2504_04704_amd import lagkv


class Counted(lagkv.Cache):
    """A cache that does something of its own for every append."""

    calls = 0

    def append_and_compress(self, K_new, V_new):
        self.calls += 1
        super().append_and_compress(K_new, V_new)


def kept(cache):
    cache._bounds[16] = [None, None, 30, 0, None]
    return cache._bounds[16]


def test_an_overriding_method_runs_once_an_append(monkeypatch):
    cache = Counted(1, 1, 64, 100, 2, 16, 0.5, device="cpu")
    cache.c.n_static, cache.c.n_tail = 10, 20
    entry, made = kept(cache), []

    def append(K_new, V_new):
        made.append((K_new, V_new))
        cache.c.n_tail += 3

    monkeypatch.setattr(cache, "_append", append, raising=False)
    cache.append_and_compress("K", "V")
    assert cache.calls == 1 and made == [("K", "V")]
    assert cache._bounds[16] is entry and entry[2] == 30      # rows behind the tail
    entry[2] = 33

    def compress(K_new, V_new):
        cache.c.n_static, cache.c.n_tail = 18, 10

    monkeypatch.setattr(cache, "_append", compress)
    cache.append_and_compress("K", "V")
    assert cache.calls == 2 and entry[2] == 10                # rows behind the static part

    def refuse(K_new, V_new):
        raise lagkv.LagKVError(lagkv.ECAPACITY, "here")

    monkeypatch.setattr(cache, "_append", refuse)
    with pytest.raises(lagkv.LagKVError):
        cache.append_and_compress("K", "V")
    assert cache.calls == 3 and cache._bounds[16] is entry and entry[2] == 10


@pytest.mark.gpu
def test_an_overriding_method_runs_once_an_append_on_the_device():
    cache = Counted(1, 1, 64, 100, 2, 16, 0.5)
    x = torch.randn(1, 1, 30, 64, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).to("cuda:0")
    cache.append_and_compress(x, x)
    cache.block_bounds(16)
    cache.append_and_compress(x, x)
    assert cache.calls == 2
