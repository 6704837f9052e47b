"""Attention over a cache in 8 bits where scales of V lie far apart and so do the weights: rows of a small scale and large weights beside, before and
behind rows of a large scale and small ones, either of which may be what the output consists of, and every tiny weight of the others may be lost but not theirs.

q and the codes of K are whole numbers and K's scales powers of two, so that q.k is exact.  With x the logits in base 2 and s the logarithm of a row's scale of V, the
exponentials are of numbers of up to max|x| + max|s| + 22 in magnitude, made by at most four roundings (d = (max|x| + max|s| + 24) 2^-22 covers them, of the logarithm too, and an
exponential's own), and three of them lie between a row and the output.  A weight is two numbers of binary16: 2^-22 of it, or 2^-35 of the largest
product of weight and scale in the row's query, for each row.  Sums as in test_attend_quantized_weights."""
import math

import pytest
import torch

from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn
TYPES = pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
CODES = pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
SCALE, COPIES = 0.25, 1200   # (as many copies as leave one piece of the cache to a workgroup: a wavefront meets first one kind of row, then the other)
BLOCK = 16


def problem(code, G, N, D, order, ratio, less, seed):
    """Rows of V's scale 1 with logits of a few units ("s") and rows of V's scale 2^ratio whose logits are some `less` lower in base 2 ("l"), 256 for each letter."""
    g = torch.Generator().manual_seed(seed)
    H, T = 1, 256 * len(order)
    whole = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g).double()  # noqa: E731
    q, K, V = whole(-1, 1, 1, G, N, D), whole(-1, 1, H, T, D), whole(-7, 7, H, T, D)
    q[..., 0] = 1.0
    K[..., 0] = 0
    K_scale, V_scale = torch.ones(H, T // BLOCK, dtype=torch.float64), torch.ones(H, T // BLOCK, dtype=torch.float64)
    step = 2.0 ** math.ceil(math.log2(max(less, 1e-3) * math.log(2) / SCALE / 15))   # (codes up to 15, which both kinds hold)
    for j, kind in enumerate(order):
        at, blocks = slice(256 * j, 256 * (j + 1)), slice(256 // BLOCK * j, 256 // BLOCK * (j + 1))
        if kind == "l":
            low = round(less * math.log(2) / SCALE / step)
            K[:, at] = 0
            K[:, at, 0] = -low - whole(0, 1, H, 256)
            K_scale[:, blocks], V_scale[:, blocks] = step, 2.0 ** ratio
    unit = 2.0 ** -max(0, min(ratio, ratio - less))    # (outputs of about 1)
    return q, K[None], V[None], K_scale[None], V_scale[None] * unit


def exact(q, K, V, K_scale, V_scale, dtype):
    u = torch.finfo(dtype).eps / 2
    k = K * K_scale.repeat_interleave(BLOCK, 2)[..., None]
    each = V_scale.repeat_interleave(BLOCK, 2)[..., None]
    v = (V * each)[0, 0]
    G, N, D = q.shape[1:]
    x = (q[0].reshape(G * N, D) @ k[0, 0].T) * SCALE
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    out = p @ v
    s = torch.log2(V_scale[V_scale > 0])
    x2, n = float(x.abs().max()) / math.log(2), k.shape[2]
    d = (x2 + float(s.abs().max()) + 24) * 2.0 ** -22
    tol = (u + 3 * d + (n + 64) * 2.0 ** -24) * out.abs() + (2.0 ** -22 + 3 * d + (n / 16 + 64) * 2.0 ** -24) * (p @ v.abs())
    tol += n * 2.0 ** -35 * (p * each[0, 0, :, 0]).amax(1, keepdim=True) * 7 + (2.0 ** -25 if dtype == HF else torch.finfo(dtype).tiny)
    tol_lse = 2 * d + (n + 64) * 2.0 ** -24 + 2.0 ** -23 * (lse.abs() + 1)
    return [t.reshape(1, G, N, *t.shape[1:]) for t in (out, lse, tol, tol_lse)]


def check(code, dtype, G, N, many, rows):
    q, K, V, K_scale, V_scale = rows
    D, T = q.shape[3], K.shape[2]
    more = lambda t: t.to(DEV).expand(COPIES, *t.shape[1:])  # noqa: E731
    x = lagkv.Quantized(more(K.to(code)), more(V.to(code)), more(K_scale.float()), more(V_scale.float()), BLOCK)
    p = lagkv.QuantParams(B=COPIES, H=1, G=G, N=N, D=D, dtype=lagkv._DTYPES[dtype], code=lagkv._CODES[code], block=BLOCK, T=T, scale=SCALE)
    plan = lagkv.attend_quantized_plan(p)[0]
    assert plan.pieces == 1 and bool(plan.many_rows) == many
    got = lagkv.attend_quantized(more(q.to(dtype)), x, scale=SCALE, want_lse=True)
    assert bool((got.out == got.out[:1]).all()) and bool((got.lse == got.lse[:1]).all())
    out, lse, tol, tol_lse = exact(*rows, dtype)
    off = abs(got.out[:1].cpu().double() - out)
    assert bool((off <= tol).all()), f"off {float((off / out.abs().amax()).max()):.2e} of the largest output, {float((off / tol).max()):.1f} of what is allowed"
    assert bool((abs(got.lse[:1].cpu().double() - lse) <= tol_lse).all())


APART = pytest.mark.parametrize("ratio,less", [(20, 10), (20, 15), (30, 20), (30, 26), (40, 26), (40, 34), (60, 50), (90, 70), (90, 85), (120, 100), (120, 112),
                                               (-20, -10), (-40, -30)], ids=lambda x: str(x))
ORDERS = pytest.mark.parametrize("order", ["sl", "ls", "sls", "ssll"])


@TYPES
@CODES
@APART
@ORDERS
def test_few_rows(order, ratio, less, code, dtype):
    for G, N, D in ((2, 2, 128), (3, 8, 64), (1, 1, 256)):
        check(code, dtype, G, N, False, problem(code, G, N, D, order, ratio, abs(less), seed=D) if ratio > 0 else mirrored(code, G, N, D, order, -ratio, -less))


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@CODES
@APART
@ORDERS
def test_many_rows(order, ratio, less, code, dtype):
    for G, N, D in ((4, 40, 128), (2, 70, 64), (3, 50, 256)):
        check(code, dtype, G, N, True, problem(code, G, N, D, order, ratio, abs(less), seed=D) if ratio > 0 else mirrored(code, G, N, D, order, -ratio, -less))


def mirrored(code, G, N, D, order, ratio, less):
    """The same with the kinds' blocks of 16 in turn within every step."""
    q, K, V, K_scale, V_scale = problem(code, G, N, D, order, ratio, less, seed=D)
    nb = K_scale.shape[2]
    turn = torch.arange(nb).reshape(2, -1).T.flatten()      # (blocks of the first and of the second half)
    rows = (turn[:, None] * BLOCK + torch.arange(BLOCK)).flatten()
    return q, K[:, :, rows], V[:, :, rows], K_scale[:, :, turn], V_scale[:, :, turn]


@pytest.mark.parametrize("G,N", [(2, 2), (4, 40)], ids=["few", "many"])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@CODES
@ORDERS
def test_scales_of_nothing(order, code, dtype, G, N):
    """Rows whose scale is 0, whatever their codes, count in the sum of the weights and add nothing else: with nearly all of the weight, or little of it."""
    for kind in "sl":
        q, K, V, K_scale, V_scale = problem(code, G, N, 128, order, 1, 30, seed=3)
        for j, c in enumerate(order):
            if c == kind:
                V_scale[:, :, 256 // BLOCK * j:256 // BLOCK * (j + 1)] = 0
        if kind == "s":
            V_scale *= 2.0 ** 28
        check(code, dtype, G, N, N > 2, (q, K, V, K_scale, V_scale))
