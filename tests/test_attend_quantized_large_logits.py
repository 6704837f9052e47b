"""Attention over a cache in 8 bits with logits so large that fp32 holds no fractions of them: each query row sees one row of the cache and nothing else of it.

q and the codes are whole numbers and K's scale a power of two, so that q.k is exact; a logit in base 2 is off by 2^-22 of itself (its factor and its rounding).  The
largest one of each query row is ahead of the next by more than that and 200, so that the weights are 1 and 0: the output is the row's value, rounded, and the logarithm the logit."""
import math

import pytest
import torch

import quant_util as Q
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn
COPIES = 1200


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("power", [10, 14, 18, 24, 40])
@pytest.mark.parametrize("apart", [0, 12], ids=["", "scales"])
@pytest.mark.parametrize("G,N,D", [(2, 2, 128), (3, 8, 64), (4, 40, 128), (3, 50, 256)], ids=str)
def test_one_row_alone(G, N, D, apart, power, dtype, code):
    T = 300
    g = torch.Generator().manual_seed(D + power)
    q = torch.randint(-3, 4, (1, G, N, D), generator=g).double()
    K = torch.randint(-15, 16, (1, 1, T, D), generator=g).double()
    V = torch.randint(-15, 16, (1, 1, T, D), generator=g).double()
    x = (q[0].reshape(G * N, D) @ K[0, 0].T)
    # (a draw that is not alone: all of it a little further from the others')
    best = x.argmax(1)
    first, second = x.topk(2, dim=1).values.T
    alone = ((first - second) * 2.0 ** power > first.abs() * 2.0 ** (power - 20) + 200) & (first > 0)
    nb = -(-T // 16)
    V_scale = 2.0 ** (torch.randint(-apart, apart + 1, (1, 1, nb), generator=g).double() / (2 if dtype == HF else 1))
    V_scale = 2.0 ** torch.log2(V_scale).round()
    copies = COPIES if G * N > 32 else 1
    more = lambda t: t.to(DEV).expand(copies, *t.shape[1:])  # noqa: E731
    y = lagkv.Quantized(more(K.to(code)), more(V.to(code)), more(torch.full((1, 1, nb), 2.0 ** power)), more(V_scale.float()), 16)
    p = lagkv.QuantParams(B=copies, H=1, G=G, N=N, D=D, dtype=lagkv._DTYPES[dtype], code=lagkv._CODES[code], block=16, T=T, scale=1.0)
    assert bool(lagkv.attend_quantized_plan(p)[0].many_rows) == (copies > 1 and dtype != FL)
    got = lagkv.attend_quantized(more(q.to(dtype)), y, scale=1.0, want_lse=True)
    assert bool((got.out == got.out[:1]).all())
    out, lse = got.out[0].cpu().double().reshape(G * N, D), got.lse[0].cpu().double().flatten()
    want = (V * V_scale.repeat_interleave(16, 2)[:, :, :T, None])[0, 0][best]
    u = torch.finfo(dtype).eps / 2
    assert int(alone.sum()) > G * N // 2
    assert bool((abs(out - want)[alone] <= (u + 2.0 ** -21) * want.abs()[alone]).all()), f"{float(abs(out - want)[alone].max()):.2e}"
    assert bool((abs(lse / (first * 2.0 ** power) - 1)[alone] <= 2.0 ** -21).all())
