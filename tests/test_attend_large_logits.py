"""Attention with logits so large that fp32 holds no fractions of them: each query row sees one row and nothing else, be it of the cache or of the new tokens, with few query
rows and many, in 16 and 32 bits and over a cache in 8 bits with a tail behind it.

q and K are whole numbers and the scale a power of two, so that a logit in base 2 is off by 2^-22 of itself; where the largest of a query row is ahead of the next by more
than that and 200 its weight is 1: the output is the row's value, rounded, and the logarithm the logit."""
import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
POWERS = pytest.mark.parametrize("power", [8, 14, 17, 18, 19, 24, 40])
SIZES = pytest.mark.parametrize("copies,G,N,D", [(1, 2, 2, 128), (1, 3, 8, 64), (1200, 4, 40, 128), (1200, 3, 50, 256), (1200, 2, 70, 64), (64, 8, 64, 128)], ids=str)


def problem(G, N, D, T, R, seed):
    g = torch.Generator().manual_seed(seed)
    whole = lambda most, *s: torch.randint(-most, most + 1, s, generator=g).double()  # noqa: E731
    return (whole(3, 1, G, N, D), *(whole(15, 1, 1, n, D) for n in (T, T, R, R, N, N)))


def check(got, q, K, V, see, power, dtype):
    """K, V: all rows in order; see [N, rows]."""
    _, G, N, D = q.shape
    out, lse = got.out[0].cpu().double(), got.lse[0].cpu().double()
    assert bool(torch.isfinite(got.out).all()) and bool((got.out == got.out[:1]).all())
    x = torch.where(see, q[0] @ K.T, -1e6)                                     # [G, N, rows]
    top, at = x.topk(2, dim=2)
    first, second = top.unbind(2)
    alone = ((first - second) * 2.0 ** power > first.abs() * 2.0 ** (power - 20) + 200) & (first > 0)
    assert int(alone.sum()) > G * N // 3
    want = V[at[..., 0]]
    u = torch.finfo(dtype).eps / 2
    assert bool((abs(out - want)[alone] <= (u + 2.0 ** -20) * want.abs()[alone]).all())
    assert bool((abs(lse / (first * 2.0 ** power) - 1)[alone] <= 2.0 ** -21).all())


@TYPES
@POWERS
@SIZES
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
def test_attend(tree, copies, G, N, D, power, dtype):
    T = 300
    q, K, V, _, _, Kn, Vn = problem(G, N, D, T, 1, D + power)
    more = lambda t: t.to(dtype).to(DEV).expand(copies, *t.shape[1:])  # noqa: E731
    parents = torch.tensor([max(-1, n - 1 - n % 3) for n in range(N)], dtype=torch.int32) if tree else None
    got = lagkv.attend(more(q), more(K), more(V), more(Kn), more(Vn), None if parents is None else parents.to(DEV), scale=2.0 ** power, want_lse=True)
    new = A.tree_visible(parents, N) if tree else torch.ones(N, N).tril().bool()
    check(got, q, torch.cat([K[0, 0], Kn[0, 0]]), torch.cat([V[0, 0], Vn[0, 0]]), torch.cat([torch.ones(N, T, dtype=torch.bool), new], 1), power, dtype)


@TYPES
@POWERS
@SIZES
@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=["int8", "e4m3"])
def test_attend_quantized(code, copies, G, N, D, power, dtype):
    T, R = 200, 90
    q, K, V, Kt, Vt, Kn, Vn = problem(G, N, D, T, R, D + power + 1)
    more = lambda t: t.to(DEV).expand(copies, *t.shape[1:])  # noqa: E731
    rows = lambda t: more(t.to(dtype))  # noqa: E731
    ones = more(torch.ones(1, 1, -(-T // 16)))
    x = lagkv.Quantized(more(K.to(code)), more(V.to(code)), ones, ones, 16)
    got = lagkv.attend_quantized(rows(q), x, rows(Kt), rows(Vt), rows(Kn), rows(Vn), scale=2.0 ** power, want_lse=True)
    see = torch.cat([torch.ones(N, T + R, dtype=torch.bool), torch.ones(N, N).tril().bool()], 1)
    check(got, q, torch.cat([K[0, 0], Kt[0, 0], Kn[0, 0]]), torch.cat([V[0, 0], Vt[0, 0], Vn[0, 0]]), see, power, dtype)
