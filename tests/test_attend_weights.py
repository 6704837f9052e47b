"""The softmax weights in the products with V: 16-bit types have them as two numbers, whichever kernel runs.

q and K hold -1, 0 and 1, so that q.k is exact.  A channel of V has two rows, 1 and -w with w the ratio of their weights for one of
the queries, rounded to the type: what is left of that query's output is far below a rounding of its weights, so that those show.
With x the logits, exp(x - m) is off by d = 2^-21 max|x| + 2^-22 of itself (the scale, in base 2, rounded, the product and
the difference rounded, the exponential to an ulp).  As two numbers of a type of unit roundoff u, of which the first leaves up to
2 u of it and the second is off by u of that, a weight is off by 2 u^2 more; where the second one is in binary16's subnormal range,
by 2^-25 in units in which the largest weight is 2^10 or more.  All rows of a channel but two add exactly 0 to its sum, which is
rounded when it is scaled anew, at most in each step of 16 rows, and joined.  The denominator, off by d and by the n + 64 roundings
of its sum, is common to all and counts by the output's own size, and so does the output's rounding."""
import math

import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
CODE = {BF: lagkv.BF16, HF: lagkv.F16, FL: lagkv.F32}


def problem(dtype, H, G, N, D, T, seed, scale=0.25):
    g = torch.Generator().manual_seed(seed)
    signs = lambda *s: torch.randint(-1, 2, s, generator=g).to(dtype)
    q, K, Kn = signs(1, H * G, N, D), signs(1, H, T, D), signs(1, H, N, D)
    V, Vn = torch.zeros(1, H, T, D, dtype=dtype), torch.zeros(1, H, N, D, dtype=dtype)
    for h in range(H):
        for c in range(D):
            i = c * 7 % (G * N)                  # the query whose output is to cancel
            x = K[0, h].double() @ q[0, h * G + i % G, i // G].double() * scale
            near = torch.randperm(T, generator=g)[:24]
            order = near[x[near].argsort()]
            up, down = int(order[-2 - c % 8]), int(order[-1])
            V[0, h, up, c] = 1.0
            V[0, h, down, c] = -torch.exp(x[up] - x[down]).to(dtype)
    return q, K, V, Kn, Vn


def exact(q, K, V, Kn, Vn, scale, parents=None, round_weights=None):
    """Outputs in 64 bits and what a kernel may be off; with round_weights the outputs of weights rounded to that type."""
    dt = q.dtype
    q, K, V, Kn, Vn = (x.double() for x in (q, K, V, Kn, Vn))
    H, N = K.shape[1], q.shape[2]
    G = q.shape[1] // H
    u = torch.finfo(dt).eps / 2
    see = A.tree_visible(parents, N) if parents is not None else torch.ones(N, N).tril().bool()
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    for hq in range(H * G):
        h = hq // G
        k, v = torch.cat([K[0, h], Kn[0, h]]), torch.cat([V[0, h], Vn[0, h]])
        x = q[0, hq] @ k.T * scale
        x[:, K.shape[2]:] = torch.where(see, x[:, K.shape[2]:], -math.inf)
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        p = e / e.sum(1, keepdim=True)
        if round_weights is not None:
            p = (e * 2.0 ** (10 if round_weights == HF else 0)).to(round_weights).double() / e.sum(1, keepdim=True) * 2.0 ** (-10 if round_weights == HF else 0)
        out[0, hq] = p @ v
        n = k.shape[0]
        d = torch.where(torch.isfinite(x), x, 0).abs().max() * 2.0 ** -21 + 2.0 ** -22
        two = 0.0 if dt == FL else 2 * u * u
        under = n * 2.0 ** -35 if dt == HF else 0.0
        tol[0, hq] = (u + d + (n + 64) * 2.0 ** -24) * out[0, hq].abs() + (two + d + (n / 16 + 24) * 2.0 ** -24) * (p @ v.abs()) + under
        tol[0, hq] += 2.0 ** -25 if dt == HF else torch.finfo(dt).tiny
    return out, tol


SIZES = [  # copies, H, G, N, D, T, tree
    (1, 2, 4, 3, 64, 300, False), (1, 1, 8, 4, 128, 260, True), (2, 1, 5, 1, 80, 700, False), (1, 1, 4, 4, 256, 200, False),
    (1, 1, 4, 2, 128, 3000, False),
    (1200, 1, 4, 30, 64, 300, False), (1200, 1, 4, 40, 128, 300, True), (1200, 1, 4, 20, 256, 200, False), (1200, 1, 3, 25, 100, 130, True),
    (8, 2, 4, 64, 128, 2000, True), (1, 4, 4, 64, 128, 9000, False),
]


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_weights_of_one_rounding_would_be_seen(dtype):
    for copies, H, G, N, D, T, tree in SIZES:
        if T <= 700 and T * N * H * G < 100000:
            args = problem(dtype, H, G, N, D, T, D + T)
            want, tol = exact(*args, 0.25)
            once, _ = exact(*args, 0.25, round_weights=dtype)
            assert int((abs(once.to(dtype).double() - want) > tol).sum()) >= D // 8, (H, G, N, D, T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_weights(size, dtype):
    copies, H, G, N, D, T, tree = size
    print("[gpu-test] weights", size, dtype, flush=True)
    x = lagkv.attend_plan(lagkv.AttendParams(copies, H, G, N, D, CODE[dtype], 0, 0, T, 0.25))
    assert bool(x.many_rows) == (copies * H * G * N > 400 and dtype != FL)
    args = problem(dtype, H, G, N, D, T, D + T)
    g = torch.Generator().manual_seed(N)
    parents = torch.tensor([int(torch.randint(max(-1, n - 6), n, (1,), generator=g)) for n in range(N)], dtype=torch.int32) if tree else None
    got = lagkv.attend(*(t.to(DEV).expand(copies, -1, -1, -1) for t in args), None if parents is None else parents.to(DEV), scale=0.25).out
    assert bool((got == got[:1]).all())
    want, tol = exact(*args, 0.25, parents)
    off = abs(got[:1].cpu().double() - want)
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.2f} of what is allowed"
