"""The operators of a cache in 8 bits on rows, codes, scales, tails and new tokens that lie more than 2^32 bytes apart, K and V different ones: by heads and batch entries
far apart, and by rows far apart."""
import pytest
import torch

from paper_2504_04704_amd import lagkv
from test_attend_quantized import BF, CODES, DEV, E4, FL, I8, rand, stored

pytestmark = pytest.mark.gpu
FAR = (1 << 32) + 4096  # bytes


def bits(t):
    return t.view(I8) if t.dtype == E4 else t


def heads_apart(t, store):
    """t [1, 2, ..] as a view of `store` with its second head FAR bytes behind the first."""
    size, far = t.element_size(), FAR // t.element_size()
    flat = store.view(t.dtype)
    inner = torch.empty(t.shape[2:], device="meta").stride()
    x = torch.as_strided(flat, t.shape, (0, far, *inner))
    bits(x).copy_(bits(t))
    assert x.stride(1) * size > 1 << 32
    return x


def rows_apart(t, store):
    """t [1, 1, rows, D] as a view of `store` in which its rows span more than 2^32 bytes."""
    step = -(-FAR // t.element_size() // (t.shape[2] - 1)) + 1
    x = torch.as_strided(store.view(t.dtype), t.shape, (0, 0, step, 1))
    bits(x).copy_(bits(t))
    assert x.stride(2) * (t.shape[2] - 1) * t.element_size() > 1 << 32
    return x


def far(tensors, way):
    """Each tensor in memory of its own."""
    return [way(t, torch.empty(FAR + (1 << 20), dtype=I8, device=DEV)) for t in tensors]


def near(way, T, D, code, seed):
    H = 2 if way is heads_apart else 1
    x = stored(1, H, T, D, 32, code, seed)
    return H, x


WAYS = pytest.mark.parametrize("way", [heads_apart, rows_apart], ids=["heads", "rows"])


@CODES
@WAYS
def test_rows_into_codes_and_back(way, code):
    T, D = 100, 64
    H, x = near(way, T, D, code, 1)
    K, V = rand(1, H, T, D, dtype=BF, seed=2), rand(1, H, T, D, dtype=BF, seed=3)
    want = lagkv.quantize(K, V, 32, code)
    k, v = far((K, V), way)
    got = lagkv.quantize(k, v, 32, code)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip((got.K, got.V, got.K_scale, got.V_scale), (want.K, want.V, want.K_scale, want.V_scale)))
    del got
    blank = [torch.zeros_like(t.view(I8)).view(t.dtype) for t in (x.K, x.V)]
    scales = [t.clone() for t in (x.K_scale, x.V_scale)]
    y = lagkv.Quantized(*far(blank, way), *(far(scales, heads_apart) if way is heads_apart else scales), 32)
    lagkv.quantize(k, v, 32, out=y)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip((y.K, y.V, y.K_scale, y.V_scale), (want.K, want.V, want.K_scale, want.V_scale)))
    back = lagkv.dequantize(want)
    k.zero_(), v.zero_()
    lagkv.dequantize(y, out=(k, v))
    assert torch.equal(k, back[0]) and torch.equal(v, back[1]) and not torch.equal(k, v)


@CODES
@pytest.mark.parametrize("dtype,N", [(BF, 1), (BF, 40), (FL, 5)], ids=["bf16-1", "bf16-40", "f32-5"])
@WAYS
def test_attention(way, dtype, N, code):
    """Few query rows, and many (as many as the kernel of many query rows takes of a few heads)."""
    T, R, D = 96, 33, 64
    H, x = near(way, T, D, code, 5)
    G = 4 if N < 40 else 40
    q = rand(1, H * G, N, D, dtype=dtype, seed=6)
    tail, new = [rand(1, H, R, D, dtype=dtype, seed=s) for s in (7, 8)], [rand(1, H, N, D, dtype=dtype, seed=s) for s in (9, 10)]
    p = lagkv.QuantParams(B=1, H=H, G=G, N=N, D=D, dtype=lagkv._DTYPES[dtype], code=lagkv._CODES[code], block=32, T=T, R=R, scale=1.0)
    assert bool(lagkv.attend_quantized_plan(p)[0].many_rows) == (N == 40)
    want = lagkv.attend_quantized(q, x, *tail, *new, want_lse=True)
    y = lagkv.Quantized(*far((x.K, x.V), way), *(far((x.K_scale, x.V_scale), heads_apart) if way is heads_apart else (x.K_scale, x.V_scale)), 32)
    far_new = far(new, way) if N > 1 or way is heads_apart else new
    got = lagkv.attend_quantized(q, y, *far(tail, way), *far_new, want_lse=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
