"""A cache whose final rows are in 8 bits, in use, beside a Cache that gets the same rows: the same rows are kept, in the same order; those in 8
bits are what quantize makes of the Cache's; attention is over what is held."""
import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I8, E4 = torch.int8, torch.float8_e4m3fn


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def same(x, cache, code):
    """x beside a Cache that got the same rows."""
    assert (x.n_static, x.n_tail, x.n_seen, x.length) == (cache.n_static, cache.n_tail, cache.n_seen, cache.length)
    assert x.n % x.rows.block == 0 and (x.n_seen < cache.S or x.window.n_static < x.rows.block)
    K, V, pos = cache.view()
    k, v, p = x.window.view()
    assert torch.equal(k, K[:, :, x.n:]) and torch.equal(v, V[:, :, x.n:]) and torch.equal(p, pos[:, :, x.n:])
    assert torch.equal(x.pos[:, :, :x.n], pos[:, :, :x.n])
    want, got = lagkv.quantize(K[:, :, :x.n], V[:, :, :x.n], x.rows.block, code), x.rows.view(x.n)
    for a, b in zip((want.K, want.V, want.K_scale, want.V_scale), (got.K, got.V, got.K_scale, got.V_scale)):
        assert torch.equal(a.view(I8) if a.dtype == E4 else a, b.view(I8) if b.dtype == E4 else b)


@pytest.mark.parametrize("dtype,D,code,block,S,L,r", [
    (torch.bfloat16, 128, I8, 16, 4, 32, 0.5), (torch.float16, 80, E4, 32, 0, 32, 0.25), (torch.float32, 64, I8, 16, 37, 16, 0.5),
    (torch.bfloat16, 128, E4, 64, 16, 128, 0.5), (torch.bfloat16, 41, I8, 16, 5, 24, 0.75)])
def test_steps_of_a_model(dtype, D, code, block, S, L, r):
    layers, B, H, G, N = 2, 2, 2, 4, 6
    x = lagkv.QuantizedCache(layers * B, H, D, 1024, S, L, r, block, code, dtype=dtype)
    cache = lagkv.Cache(layers * B, H, D, 1200, S, L, r, dtype=dtype)
    T = 700
    K, V = rand(layers * B, H, T, D, dtype=dtype, seed=1), rand(layers * B, H, T, D, dtype=dtype, seed=2)
    assert x.prefill_chunked(K, V) == cache.prefill_chunked(K, V)
    same(x, cache, code)
    assert x.n > 0
    parents = torch.tensor([-1, 0, 0, 1, 3, 2], dtype=torch.int32, device=DEV)
    path = [0, 1, 3, 4]                                        # what the model accepts of every tree
    grown = 0
    for step in range(40):
        Kn, Vn = rand(layers * B, H, N, D, dtype=dtype, seed=100 + step), rand(layers * B, H, N, D, dtype=dtype, seed=200 + step)
        for layer in range(layers):
            at = slice(layer * B, (layer + 1) * B)
            q = rand(B, N, H * G, D, dtype=dtype, seed=300 + step + 50 * layer).transpose(1, 2)
            got = x.attend(q, Kn[at], Vn[at], parents, batch=at, want_lse=True)
            if step % 10 == 0:
                k, v, _ = x.window.view()
                A.check(got, Q.attend(q, x.rows.view(x.n, at), k[at], v[at], Kn[at], Vn[at], parents), f"step {step}")
        n = x.n
        x.append_and_compress(Kn[:, :, path], Vn[:, :, path])
        cache.append_and_compress(Kn[:, :, path], Vn[:, :, path])
        grown += x.n > n
        same(x, cache, code)
    assert grown >= 1
    k, v, p = x.view()
    assert k.shape == cache.view()[0].shape and torch.equal(p, cache.view()[2])
    back = lagkv.dequantize(x.rows.view(x.n), dtype)
    assert torch.equal(k[:, :, :x.n], back[0]) and torch.equal(v[:, :, x.n:], cache.view()[1][:, :, x.n:])


@pytest.mark.parametrize("T", [3, 20, 90, 1000])
def test_from_compressed(T):
    """What compress() makes of a prompt shorter than its sink, than what is compressed, and longer; rows appended behind it."""
    S, L, r, block = 10, 32, 0.5, 16
    K, V = rand(2, 2, T, 64, dtype=torch.bfloat16, seed=3), rand(2, 2, T, 64, dtype=torch.bfloat16, seed=4)
    comp = lagkv.compress(K, V, S, L, r)
    x = lagkv.QuantizedCache.from_compressed(comp, T, 1024, S, L, r, block)
    cache = lagkv.Cache.from_compressed(comp, T, 1500, S, L, r)
    same(x, cache, I8)
    for step, n in enumerate([1, 5, 30, 0, 64, 7]):
        Kn, Vn = rand(2, 2, n, 64, dtype=torch.bfloat16, seed=10 + step), rand(2, 2, n, 64, dtype=torch.bfloat16, seed=20 + step)
        x.append_and_compress(Kn, Vn)
        cache.append_and_compress(Kn, Vn)
        same(x, cache, I8)
    q = rand(2, 4, 1, 64, dtype=torch.bfloat16, seed=5)
    k, v, _ = x.window.view()
    A.check(x.attend(q, want_lse=True), Q.attend(q, x.rows.view(x.n), k, v))


def test_no_room_in_8_bits():
    """Blocks that do not fit stay in the window, until it is full as well: then an append is refused, and changes nothing."""
    S, L, r = 0, 16, 1.0
    x = lagkv.QuantizedCache(1, 1, 32, 40, S, L, r, 16, window=80)
    cache = lagkv.Cache(1, 1, 32, 400, S, L, r)
    refused = 0
    for step in range(12):
        Kn, Vn = rand(1, 1, 16, 32, dtype=torch.bfloat16, seed=step), rand(1, 1, 16, 32, dtype=torch.bfloat16, seed=50 + step)
        before = (x.n, x.length, x.n_seen)
        try:
            x.append_and_compress(Kn, Vn)
        except lagkv.LagKVError as e:
            assert e.status == lagkv.ECAPACITY and (x.n, x.length, x.n_seen) == before
            refused += 1
            continue
        cache.append_and_compress(Kn, Vn)
        assert x.length == cache.length and x.n <= 32
        assert torch.equal(x.window.view()[0], cache.view()[0][:, :, x.n:])
    assert refused > 0 and x.n == 32 and x.length == 32 + 80
    with pytest.raises(lagkv.LagKVError):
        lagkv.QuantizedCache.from_compressed(lagkv.compress(*(rand(1, 1, 500, 32, dtype=torch.bfloat16, seed=9),) * 2, S, L, 0.5), 500, 64, S, L, 0.5, 16)


def test_without_positions():
    x = lagkv.QuantizedCache(1, 2, 64, 256, 4, 32, 0.5, 16, track_positions=False)
    x.prefill_chunked(rand(1, 2, 300, 64, dtype=torch.bfloat16, seed=1), rand(1, 2, 300, 64, dtype=torch.bfloat16, seed=2))
    assert x.pos is None and x.view()[2] is None and x.n > 0
