"""Attention over a cache in 8 bits by the kernel that many query rows share, in every form that it has, named by the plan of the call."""
import math

import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv
from test_attend_quantized import BF, CODES, DEV, E4, HF, I8, problem, tree

pytestmark = pytest.mark.gpu
MANY = 1200  # copies of a problem, for which the kernel is taken at small shapes (their strides along the batch are 0)


def copies(*tensors):
    return [None if t is None else t[:1].expand(MANY, *t.shape[1:]) for t in tensors]


def many(x):
    return lagkv.Quantized(*copies(x.K, x.V, x.K_scale, x.V_scale), x.block)


def plan(q, x, R):
    B, H, T, D = x.K.shape
    p = lagkv.QuantParams(B=B, H=H, G=q.shape[1] // H, N=q.shape[2], D=D, dtype=lagkv._DTYPES[q.dtype], code=lagkv._CODES[x.K.dtype], block=x.block,
                          T=T, R=R, scale=1.0)
    return lagkv.attend_quantized_plan(p)[0]


def the_first_of(got):
    """The first copy's result; that of all the others is the same, bit for bit."""
    assert bool((got.out.nan_to_num(7.0) == got.out[:1].nan_to_num(7.0)).all())
    assert bool((got.lse.nan_to_num(7.0) == got.lse[:1].nan_to_num(7.0)).all())
    return lagkv.Attended(got.out[:1].clone(), got.lse[:1].clone())


def of_many(q, x, Kt, Vt, Kn, Vn, parents=None, **kw):
    x, R = many(x), 0 if Kt is None else Kt.shape[2]
    q, Kt, Vt, Kn, Vn = copies(q, Kt, Vt, Kn, Vn)
    assert plan(q, x, R).many_rows == 1
    return the_first_of(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, parents, want_lse=True, **kw))


SIZES = [  # H, G, N, D, T, R, new, block
    (1, 1, 70, 128, 20, 7, "tree", 16), (1, 3, 50, 128, 100, 31, "chain", 64), (2, 4, 40, 128, 700, 90, "tree", 64),
    (1, 2, 130, 64, 129, 33, "chain", 16), (1, 3, 30, 40, 100, 12, "tree", 32), (1, 7, 21, 100, 230, 50, "chain", 32),
    (1, 4, 20, 200, 150, 20, "tree", 16), (1, 2, 65, 256, 61, 60, "chain", 32), (1, 4, 30, 128, 300, 0, "none", 16),
    (1, 5, 60, 128, 390, 10, "chain", 1024), (1, 2, 20, 17, 64, 0, "none", 64), (1, 8, 16, 96, 1, 0, "chain", 16),
    (1, 2, 64, 128, 64, 5, "chain", 32), (1, 2, 100, 128, 64 * 6 + 1, 5, "chain", 32), (1, 2, 90, 72, 130, 70, "chain", 32),
    (1, 1, 150, 104, 64, 200, "tree", 16), (1, 2, 40, 245, 40, 3, "chain", 16), (1, 4, 50, 128, 3, 500, "chain", 16),
]


def test_forms():
    """The sizes reach every form: up to 64, 128 and 256 channels."""
    forms = set()
    for H, G, N, D, T, R, new, block in SIZES:
        p = lagkv.QuantParams(B=MANY, H=H, G=G, N=N, D=D, dtype=lagkv.BF16, block=block, T=T, R=R, scale=1.0)
        got = lagkv.attend_quantized_plan(p)[0]
        assert got.many_rows
        forms.add((64 if D <= 64 else 128 if D <= 128 else 256, got.row_tile))
    assert forms == {(64, 128), (128, 128), (256, 128)}


@CODES
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_of_many_streams(size, dtype, code):
    H, G, N, D, T, R, new, block = size
    print("[gpu-test] attend_quantized, many streams", size, dtype, code, flush=True)
    q, x, *rows = problem(dtype, code, 1, H, G, N, D, T, R, new, block, seed=D + T)
    parents = tree(N, T) if new == "tree" else None
    A.check(of_many(q, x, *rows, parents), Q.attend(q, x, *rows, parents), str(size))


@CODES
@pytest.mark.parametrize("size", [(4, 8, 4, 64, 128, 2100, 40, "tree"), (1, 8, 4, 150, 256, 2000, 0, "chain"), (2, 4, 8, 200, 100, 3000, 70, "chain"),
                                  (2, 4, 4, 200, 64, 6001, 5, "chain")], ids=lambda s: "x".join(map(str, s)))
def test_of_long_caches(size, code):
    B, H, G, N, D, T, R, new = size
    q, x, Kt, Vt, Kn, Vn = problem(BF, code, B, H, G, N, D, T, R, new, 64, seed=D + T)
    parents = tree(N, T, B) if new == "tree" else None
    got = plan(q, x, R)
    assert got.many_rows == 1 and got.pieces > 1
    got = lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, parents, want_lse=True)
    for b in range(B):  # (every few heads of every batch entry)
        for i in (0, H * G // 2, H * G - 1):
            pick = lambda t, j: None if t is None else t[b:b + 1, j:j + 1]
            y = lagkv.Quantized(*(pick(t, i // G) for t in (x.K, x.V, x.K_scale, x.V_scale)), 64)
            want = Q.attend(pick(q, i), y, *(pick(t, i // G) for t in (Kt, Vt, Kn, Vn)), None if parents is None else parents[b:b + 1])
            A.check(lagkv.Attended(pick(got.out, i), pick(got.lse, i)), want, f"{b} {i}")


@CODES
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_lengths(D, dtype, code):
    """Lengths as of few rows, 150 times each; what lies behind is no number."""
    N, T, R = 20, 200, 30
    lens, tails = [0, 1, 64, 65, 127, 200, 1000, -7], [0, 30, 1, 0, 17, 99, 5, 30]
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, len(lens), 2, 4, N, D, T, R, "chain", 32, seed=3)
    lengths, tail_lengths = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (lens, tails))
    want = Q.attend(q, x, Kt, Vt, Kn, Vn, None, lengths, tail_lengths)
    for b, (n, k) in enumerate(zip(lens, tails)):
        n, k = min(max(n, 0), T), min(max(k, 0), R)
        x.K.view(I8)[b, :, n:], x.V.view(I8)[b, :, n:] = -1, 127
        x.K_scale[b, :, -(-n // 32):], x.V_scale[b, :, -(-n // 32):] = math.nan, math.inf
        Kt[b, :, k:], Vt[b, :, k:] = math.nan, math.inf
    r = lambda t: None if t is None else t.repeat(150, *[1] * (t.dim() - 1))
    c = lambda t: r(t.view(I8)).view(t.dtype)
    y = lagkv.Quantized(c(x.K), c(x.V), r(x.K_scale), r(x.V_scale), 32)
    assert plan(r(q), y, R).many_rows == 1
    got = lagkv.attend_quantized(r(q), y, r(Kt), r(Vt), r(Kn), r(Vn), None, r(lengths), r(tail_lengths), want_lse=True)
    A.check(lagkv.Attended(got.out[:8], got.lse[:8]), want)
    assert torch.equal(got.out, r(got.out[:8])) and torch.equal(got.lse, r(got.lse[:8]))


@CODES
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_scales_and_queries_of_all_sizes(dtype, code):
    N, T = 40, 330
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, 1, 1, 3, N, 128, T, 20, "chain", 16, seed=21)
    nb = x.V_scale.shape[2]
    for lo, hi in ((-30, 30), (30, -30), (-30, -28), (-2, 2), (2, -2)):
        if dtype == HF and max(lo, hi) > 2:
            continue  # (the outputs would not fit)
        x.V_scale.copy_((10 ** torch.linspace(lo, hi, nb)).to(DEV).expand_as(x.V_scale))
        x.V_scale[:, :, nb // 3] = 0
        A.check(of_many(q, x, Kt, Vt, Kn, Vn), Q.attend(q, x, Kt, Vt, Kn, Vn), str((lo, hi)))
    x.V_scale.fill_(0.01)
    x.K_scale[0, 0, 3], x.K_scale[0, 0, nb - 1] = 0, 0          # (the last block is one that is not whole)
    q = q.contiguous()
    x.K.view(I8)[..., 7] = 0
    Kt[..., 7], Kn[..., 7] = 0, 0
    q[:, 0, ::2, 7], q[:, 1, ::3], q[0, 2, 1] = 30000.0, 0, torch.finfo(dtype).tiny
    A.check(of_many(q, x, Kt, Vt, Kn, Vn), Q.attend(q, x, Kt, Vt, Kn, Vn))
    for scale in (0.0, -0.3, 1.0):
        A.check(of_many(q, x, Kt, Vt, Kn, Vn, scale=scale), Q.attend(q, x, Kt, Vt, Kn, Vn, scale=scale), str(scale))


@CODES
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("T", [64, 300])
def test_what_is_no_number_and_is_seen(T, dtype, code):
    N = 40
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, 1, 2, 3, N, 128, T, 20, "chain", 16, seed=31)
    want = Q.attend(q, x, Kt, Vt, Kn, Vn)

    def nan_in(got, bad):
        assert bool(torch.isnan(got.out[0, bad]).all()) and bool(torch.isnan(got.lse[0, bad]).all())
        got.out[0, bad], got.lse[0, bad] = want[0][0, bad].to(dtype).to(DEV), want[1][0, bad].float().to(DEV)
        A.check(got, want)

    for value in (math.nan, math.inf, -math.inf):
        q2 = q.clone()
        q2[0, 4, N - 1, 5] = value
        bad = torch.zeros(6, N, dtype=torch.bool)
        bad[4, N - 1] = True
        nan_in(of_many(q2, x, Kt, Vt, Kn, Vn), bad)
    bad = torch.zeros(6, N, dtype=torch.bool)
    bad[3:] = True
    for block in (T // 32, -1):  # (the last one is not whole where T is 300)
        keep = x.K_scale.clone()
        x.K_scale[0, 1, block] = math.nan
        nan_in(of_many(q, x, Kt, Vt, Kn, Vn), bad)
        x.K_scale.copy_(keep)
    if code == E4:
        was = x.K.view(I8)[0, 1, T - 1, 9].item()
        x.K.view(I8)[0, 1, T - 1, 9] = 127
        nan_in(of_many(q, x, Kt, Vt, Kn, Vn), bad)
        x.K.view(I8)[0, 1, T - 1, 9] = was
        x.V.view(I8)[0, 1, T - 1, 9] = -1
        got = of_many(q, x, Kt, Vt, Kn, Vn)
        assert bool(torch.isnan(got.out[0, 3:, :, 9]).all())
        got.out[0, 3:, :, 9] = want[0][0, 3:, :, 9].to(dtype).to(DEV)
        A.check(got, want)
    x.V_scale[0, 0, -1] = math.nan
    got = of_many(q, x, Kt, Vt, Kn, Vn)
    assert bool(torch.isnan(got.out[0, :3]).all()) and bool(torch.isfinite(got.lse).all())
