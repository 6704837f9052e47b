"""The operators that read a cache give the same through the native binding and through ctypes, and through ctypes refuse the same."""
import pytest
import torch

from paper_2504_04704_amd import lagkv

DEV = "cuda:0"


def rand(*shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("N,T", [(1, 50), (5, 3000), (40, 900), (3, 0), (0, 20)])
def test_both_paths(N, T, monkeypatch):
    B, H, G, D, block, k = 2, 2, 4, 72, 16, 6
    q, K, V, Kn, Vn = rand(B, H * G, N, D, seed=1), rand(B, H, T, D, seed=2), rand(B, H, T, D, seed=3), rand(B, H, N, D, seed=4), rand(B, H, N, D, seed=5)
    lengths = torch.tensor([T, T // 2], dtype=torch.int32, device=DEV)
    parents = torch.tensor([n - 1 - n % 2 for n in range(N)], dtype=torch.int32, device=DEV).clamp(min=-1)

    def step():
        lo, hi = lagkv.block_bounds(K, block, lengths)
        blocks = lagkv.select_blocks(q, lo, hi, T, block, k, 1, 2, lengths)
        some = lagkv.attend_blocks(q, K, V, blocks, block, Kn, Vn, parents, lengths, want_lse=True)
        every = lagkv.attend(q, K, V, Kn, Vn, parents, lengths, scale=0.2, want_lse=True)
        alone = lagkv.attend(q, K, V, want_lse=True)             # (rows of the cache alone: none, with T = 0)
        return lo, hi, blocks, some.out, some.lse, every.out, every.lse, alone.out, alone.lse

    lagkv.load()
    assert lagkv._native is not None
    native = step()
    monkeypatch.setattr(lagkv, "_native", None)
    for a, b in zip(native, step()):
        assert a.shape == b.shape and torch.equal(a, b)
    if T == 0:
        assert bool((native[-2] == 0).all()) and bool((native[-1] == -float("inf")).all())
    w = q.clone().requires_grad_()
    for f in (lambda: lagkv.attend(w, K, V), lambda: lagkv.select_blocks(w, native[0], native[1], T, block, k)):
        with pytest.raises(RuntimeError, match="no backward"):
            f()
    with pytest.raises(lagkv.LagKVError):
        lagkv.attend_blocks(q, K, V, native[2], 17)
