"""Attention over a cache in 8 bits: a query's elements go into the products with K as they are, however far below the row's largest they lie.  Channel 0 has the
largest of q and nothing of K; the others' elements are up to 2^-24 of it, with as many bits as the type has, and meet keys large enough to matter.  Bounds are those
of the same rows in attention over 16 or 32 bits, without anything for q."""
import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn
COPIES = 1200


def problem(dtype, code, G, N, D, T, below, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((1, G, N, D), generator=g) * 2.0 ** -below
    q[..., 0] = torch.where(torch.arange(G * N).reshape(1, G, N) % 2 == 0, 1.5, -1.25)
    codes = (torch.randn((1, 1, T, D), generator=g) * 30).round().clamp(-127, 127) if code == I8 else torch.randn((1, 1, T, D), generator=g) * 60
    codes[..., 0] = 0
    V = (torch.randn((1, 1, T, D), generator=g) * 30).round().clamp(-127, 127)
    nb = -(-T // 16)
    each = torch.exp(0.5 * torch.randn((2, 1, 1, nb), generator=g)) * torch.tensor([2.0 ** (below - 5), 0.02]).reshape(2, 1, 1, 1)
    return q.to(dtype), codes.to(code), V.to(code), each[0], each[1]


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("below", [0, 12, 18, 24])
@pytest.mark.parametrize("G,N,D", [(2, 2, 128), (3, 8, 64), (1, 3, 41), (1, 2, 256), (3, 30, 128), (2, 50, 64), (4, 20, 256)], ids=str)
def test_small_elements(G, N, D, below, dtype, code):
    q, K, V, K_scale, V_scale = problem(dtype, code, G, N, D, 200, below, seed=D + below)
    x = lagkv.Quantized(K, V, K_scale, V_scale, 16)
    copies = COPIES if G * N > 32 else 1
    more = lambda t: t.to(DEV).expand(copies, *t.shape[1:])  # noqa: E731
    y = lagkv.Quantized(*(more(t) for t in (K, V, K_scale, V_scale)), 16)
    p = lagkv.QuantParams(B=copies, H=1, G=G, N=N, D=D, dtype=lagkv._DTYPES[dtype], code=lagkv._CODES[code], block=16, T=200, scale=1.0)
    assert bool(lagkv.attend_quantized_plan(p)[0].many_rows) == (copies > 1 and dtype != FL)
    got = lagkv.attend_quantized(more(q), y, want_lse=True)
    assert bool((got.out == got.out[:1]).all()) and bool((got.lse == got.lse[:1]).all())
    want = A.attend(q, Q.values(x.K, x.K_scale, 16), Q.values(x.V, x.V_scale, 16))
    A.check(lagkv.Attended(got.out[:1], got.lse[:1]), want, f"{below}")
