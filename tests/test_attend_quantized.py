"""Attention over a cache in 8 bits, a tail that is not quantised and new tokens, against the plain 64-bit form over the rows that the codes
stand for."""
import math

import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn
CODES = pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
TYPES = pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])


def rand(*shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def stored(B, H, T, D, block, code, seed, k=1.5, v=1.0):
    """A cache of T rows in 8 bits, with scales that differ from block to block and codes made here (not by quantize)."""
    g = torch.Generator().manual_seed(seed)
    nb = -(-T // block)
    out = []
    for top in (k, v):
        x = torch.randn((B, H, T, D), generator=g)
        each = torch.exp(0.7 * torch.randn((B, H, nb), generator=g)) * (top / (40.0 if code == I8 else 100.0))
        x = x * (40.0 if code == I8 else 100.0)
        codes = x.round().clamp(-127, 127).to(I8) if code == I8 else x.clamp(-448, 448).to(E4)
        out.append((codes.to(DEV), each.float().to(DEV)))
    return lagkv.Quantized(out[0][0], out[1][0], out[0][1], out[1][1], block)


def problem(dtype, code, B, H, G, N, D, T, R, new, block=32, seed=0):
    q = rand(B, N, H * G, D, dtype=dtype, seed=seed).transpose(1, 2)
    x = stored(B, H, T, D, block, code, seed + 1)
    Kt, Vt = (rand(B, H, R, D, dtype=dtype, seed=seed + 2, scale=1.5), rand(B, H, R, D, dtype=dtype, seed=seed + 3)) if R else (None, None)
    Kn, Vn = (rand(B, H, N, D, dtype=dtype, seed=seed + 4), rand(B, H, N, D, dtype=dtype, seed=seed + 5)) if new != "none" else (None, None)
    return q, x, Kt, Vt, Kn, Vn


def tree(N, seed, B=None, padded=0):
    g = torch.Generator().manual_seed(seed)
    rows = []
    for _ in range(B or 1):
        p = [int(torch.randint(max(-1, n - 6), n, (1,), generator=g)) for n in range(N)]
        for i in range(padded):
            p[N - 1 - i] = -2 if i % 2 == 0 else 1000
        rows.append(p)
    t = torch.tensor(rows, dtype=torch.int32, device=DEV)
    return t if B else t[0]


SIZES = [  # B, H, G, N, D, T, R, new, block
    (1, 1, 1, 1, 64, 1, 0, "none", 16),
    (1, 2, 2, 1, 64, 0, 5, "chain", 16),
    (2, 1, 3, 1, 128, 31, 1, "chain", 16),
    (1, 2, 4, 1, 128, 65, 33, "chain", 32),
    (2, 2, 8, 1, 80, 257, 0, "none", 64),
    (1, 1, 5, 7, 96, 130, 20, "tree", 128),
    (2, 2, 4, 8, 128, 515, 64, "tree", 32),    # 32 query rows
    (1, 2, 4, 9, 128, 300, 100, "tree", 16),   # 36
    (1, 1, 2, 33, 64, 65, 0, "tree", 1024),
    (1, 1, 1, 70, 128, 20, 7, "tree", 16),
    (1, 1, 3, 50, 128, 100, 31, "chain", 64),
    (1, 1, 2, 1, 256, 100, 40, "chain", 16),
    (1, 2, 3, 5, 256, 77, 3, "tree", 32),
    (1, 1, 2, 3, 16, 50, 9, "chain", 16),      # the narrowest head
    (1, 2, 2, 2, 41, 90, 17, "tree", 32),      # rows on odd addresses
    (1, 1, 4, 2, 100, 70, 64, "tree", 16),
    (1, 1, 6, 3, 250, 40, 2, "chain", 64),
    (1, 1, 1, 1, 128, 3000, 200, "chain", 64),  # the cache in pieces
    (1, 1, 4, 16, 128, 2500, 130, "tree", 128),
    (2, 1, 130, 1, 64, 90, 30, "chain", 16),   # more query heads than a tile
    (1, 2, 4, 40, 128, 700, 90, "tree", 64),   # many query rows
    (1, 1, 5, 60, 128, 190, 10, "chain", 32),
    (1, 1, 2, 130, 64, 129, 33, "chain", 16),
    (1, 1, 3, 12, 41, 100, 12, "tree", 16),
    (1, 2, 7, 21, 100, 230, 50, "chain", 32),
    (1, 1, 4, 20, 250, 150, 20, "tree", 16),
    (1, 1, 2, 65, 256, 60, 60, "chain", 32),
    (1, 1, 8, 16, 128, 3000, 70, "tree", 64),
]


@CODES
@TYPES
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_attend_quantized(size, dtype, code):
    B, H, G, N, D, T, R, new, block = size
    print("[gpu-test] attend_quantized", size, dtype, code, flush=True)
    q, x, *rows = problem(dtype, code, B, H, G, N, D, T, R, new, block, seed=D + T)
    parents = tree(N, T, B) if new == "tree" else None
    got = lagkv.attend_quantized(q, x, *rows, parents, want_lse=True)
    assert got.out.stride() == q.stride()
    A.check(got, Q.attend(q, x, *rows, parents), str(size))


@CODES
@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", ["none", "chain", "tree"])
@pytest.mark.parametrize("N,T", [(5, 200), (20, 200), (1, 5000)])
def test_ragged_lengths_and_what_lies_behind_them(N, T, new, dtype, code):
    """Lengths of nothing, of one row, inside and at the end of a step, a block and a piece, and beyond the rows there are; what lies behind
    them holds codes, scales and rows that are no numbers."""
    if new == "tree" and N == 1:
        pytest.skip("a tree of one token is a chain of one")
    lens, tails = [0, 1, 16, 33, 100, 200, 10 * T, -7, 0, T - 1], [0, 40, 0, 1, 16, 39, 1000, 7, 33, -1]
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, len(lens), 2, 4, N, 64, T, 40, new, 32, seed=3)
    lengths, tail_lengths = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (lens, tails))
    parents = tree(N, 1, len(lens), padded=2 if N > 8 else 0) if new == "tree" else None
    want = Q.attend(q, x, Kt, Vt, Kn, Vn, parents, lengths, tail_lengths)
    for b, (n, r) in enumerate(zip(lens, tails)):
        n, r = min(max(n, 0), T), min(max(r, 0), 40)
        x.K.view(I8)[b, :, n:], x.V.view(I8)[b, :, n:] = -1, 127
        x.K_scale[b, :, -(-n // 32):], x.V_scale[b, :, -(-n // 32):] = math.nan, math.inf
        Kt[b, :, r:], Vt[b, :, r:] = math.nan, math.inf
    got = lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, parents, lengths, tail_lengths, want_lse=True)
    A.check(got, want)
    if new == "none":
        assert bool((got.out[0] == 0).all()) and bool((got.lse[0] == -math.inf).all())


@CODES
@TYPES
@pytest.mark.parametrize("size", [(1, 1, 8, 1, 128, 60001, 300), (1, 3, 4, 9, 128, 7000, 64), (1, 7, 32, 1, 100, 3001, 0), (1, 1, 2, 17, 256, 9000, 99)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_pieces_of_few_streams(size, dtype, code):
    B, H, G, N, D, T, R = size
    q, x, *rows = problem(dtype, code, B, H, G, N, D, T, R, "chain", 64, seed=T)
    A.check(lagkv.attend_quantized(q, x, *rows, want_lse=True), Q.attend(q, x, *rows))


@CODES
@TYPES
@pytest.mark.parametrize("T,N", [(200, 1), (200, 12), (3000, 3)])
def test_scales_of_all_sizes(T, N, dtype, code):
    """Scales of V from block to block 1e-30 to 1e30 (in either order), of 0, and of K with queries that make up for them."""
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, 2, 1, 3, N, 64, T, 20, "chain", 16, seed=21)
    g = torch.Generator().manual_seed(4)
    nb = x.V_scale.shape[2]
    for lo, hi in ((-30, 30), (-30, -28), (-2, 2), (25, 30), (-44, -38), (35.5, 35.5)):
        if dtype == HF and hi > 2:
            continue  # (the outputs would not fit)
        powers = torch.linspace(lo, hi, nb)
        x.V_scale.copy_(torch.stack([10 ** powers, 10 ** powers.flip(0)])[:, None].to(DEV))
        x.V_scale[:, :, nb // 3] = 0
        got = lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True)
        A.check(got, Q.attend(q, x, Kt, Vt, Kn, Vn), str((lo, hi)))
    if dtype != HF:
        x.V_scale.fill_(0.01)
        up = torch.exp(torch.rand(nb, generator=g)).to(DEV) * 1e-2
        for f in (1e-25, 1e25):
            x.K_scale.copy_((up * f).expand_as(x.K_scale))
            zero = torch.zeros_like
            got = lagkv.attend_quantized((q.float() / f).to(dtype), x, zero(Kt), Vt, zero(Kn), Vn, want_lse=True)
            A.check(got, Q.attend((q.float() / f).to(dtype), x, zero(Kt), Vt, zero(Kn), Vn), str(f))


@CODES
@TYPES
def test_queries_of_all_sizes(dtype, code):
    """A query row with one channel that dwarfs the others, which the cache's rows hold 0 in; rows of zeros and of the smallest numbers."""
    N = 4
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, 1, 2, 2, N, 96, 300, 10, "chain", 32, seed=22)
    q = q.contiguous()
    x.K.view(I8)[..., 7] = 0
    Kt[..., 7], Kn[..., 7] = 0, 0
    q[:, 0, :, 7] = 30000.0
    q[:, 1] = 0
    q[:, 2] *= 1e-6
    q[0, 3, 0] = torch.finfo(dtype).tiny
    A.check(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True), Q.attend(q, x, Kt, Vt, Kn, Vn))


@CODES
@TYPES
@pytest.mark.parametrize("N,T", [(1, 64), (1, 3000), (24, 64), (24, 3000)])
def test_what_is_no_number_and_is_seen(N, T, dtype, code):
    """A query with NaN or an infinity, a scale or a code that is none: the outputs that see it are none, and no others."""
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
        nan_in(lagkv.attend_quantized(q2, x, Kt, Vt, Kn, Vn, want_lse=True), bad)
    bad = torch.zeros(6, N, dtype=torch.bool)
    bad[3:] = True
    keep = x.K_scale.clone()
    x.K_scale[0, 1, T // 32] = math.nan
    nan_in(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True), bad)
    x.K_scale.copy_(keep)
    if code == E4:
        was = x.K.view(I8)[0, 1, T // 2, 9].item()
        x.K.view(I8)[0, 1, T // 2, 9] = 127
        nan_in(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True), bad)
        x.K.view(I8)[0, 1, T // 2, 9] = was
        x.V.view(I8)[0, 1, T // 2, 9] = -1
        got = lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True)
        assert bool(torch.isnan(got.out[0, 3:, :, 9]).all())
        got.out[0, 3:, :, 9] = want[0][0, 3:, :, 9].to(dtype).to(DEV)
        A.check(got, want)
        x.V.view(I8)[0, 1, T // 2, 9] = 0
    x.V_scale[0, 0, T // 32] = math.nan
    got = lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True)
    assert bool(torch.isnan(got.out[0, :3]).all()) and bool(torch.isfinite(got.lse).all()) and bool(torch.isfinite(got.out[0, 3:]).all())


def test_padded_trees():
    N = 12
    q, x, Kt, Vt, Kn, Vn = problem(BF, I8, 3, 2, 2, N, 128, 60, 10, "tree", 16, seed=4)
    parents = tree(N, 8, 3, padded=4)
    parents[1, 0] = -5
    parents[2, 3] = 3
    want = Q.attend(q, x, Kt, Vt, Kn, Vn, parents)
    q = q.contiguous()
    for b in range(3):
        for n in range(N):
            if int(parents[b, n]) < -1 or int(parents[b, n]) >= n:
                Kn[b, :, n], Vn[b, :, n], q[b, :, n] = math.nan, math.nan, math.nan
    A.check(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, parents, want_lse=True), want)


@CODES
@TYPES
def test_strides(dtype, code):
    """Codes in a larger store with room behind and between, on odd addresses; scales with room; a tail that is a slice of a cache; an output
    between rows that stay as they were."""
    B, H, G, N, D, T, R = 2, 3, 2, 4, 72, 90, 21
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, B, H, G, N, D, T, R, "chain", 32, seed=12)
    want = Q.attend(q, x, Kt, Vt, Kn, Vn)
    store = torch.full((2, B, 100, H, D + 5), -1, dtype=I8, device=DEV)
    scales = torch.full((2, B, H + 1, 9), math.nan, device=DEV)
    big = torch.full((2, B, H, 60, D), math.nan, dtype=dtype, device=DEV)
    for i, (c, s, t) in enumerate(((x.K, x.K_scale, Kt), (x.V, x.V_scale, Vt))):
        store[i, :, 5:5 + T, :, 3:3 + D] = c.view(I8).transpose(1, 2)
        scales[i, :, :H, 2:5] = s
        big[i, :, :, 10:10 + R] = t
    y = lagkv.Quantized(*(store[i].view(code)[:, 5:5 + T, :, 3:3 + D].transpose(1, 2) for i in range(2)),
                        *(scales[i, :, :H, 2:5] for i in range(2)), 32)
    out = torch.full((B, N, H * G + 1, D + 3), 7.0, dtype=dtype, device=DEV)
    view = out[:, :, 1:, 1:1 + D].transpose(1, 2)
    got = lagkv.attend_quantized(q, y, big[0, :, :, 10:10 + R], big[1, :, :, 10:10 + R], Kn, Vn, out=view, want_lse=True)
    assert got.out is view
    A.check(got, want)
    assert bool((out[:, :, 0] == 7.0).all()) and bool((out[..., 0] == 7.0).all()) and bool((out[..., 1 + D:] == 7.0).all())
    same = q.clone(memory_format=torch.preserve_format)
    A.check(lagkv.attend_quantized(same, x, Kt, Vt, Kn, Vn, out=same, want_lse=True), want)
    one = lagkv.Quantized(x.K[:1].expand(B, H, T, D), x.V[:1].expand(B, H, T, D), x.K_scale[:1].expand(B, H, 3), x.V_scale[:1].expand(B, H, 3), 32)
    A.check(lagkv.attend_quantized(q, one, Kt, Vt, Kn, Vn, want_lse=True), Q.attend(q, one, Kt, Vt, Kn, Vn))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0, 1e-3])
def test_scale_of_the_logits(scale):
    for dtype in (BF, FL):
        q, x, Kt, Vt, Kn, Vn = problem(dtype, E4, 1, 2, 2, 5, 64, 150, 30, "chain", 32, seed=13)
        A.check(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, scale=scale, want_lse=True), Q.attend(q, x, Kt, Vt, Kn, Vn, scale=scale))


def test_rows_that_were_quantised():
    """quantize, dequantize, attend and attend_quantized over the same rows, as a program uses them together."""
    for code in (I8, E4):
        K, V = rand(2, 2, 333, 128, dtype=BF, seed=1), rand(2, 2, 333, 128, dtype=BF, seed=2)
        q, Kn, Vn = rand(2, 8, 3, 128, dtype=BF, seed=3), rand(2, 2, 3, 128, dtype=BF, seed=4), rand(2, 2, 3, 128, dtype=BF, seed=5)
        x = lagkv.quantize(K[:, :, :256], V[:, :, :256], 64, code)
        got = lagkv.attend_quantized(q, x, K[:, :, 256:], V[:, :, 256:], Kn, Vn, want_lse=True)
        A.check(got, Q.attend(q, x, K[:, :, 256:], V[:, :, 256:], Kn, Vn))
        want = Q.attend(q, x, K[:, :, 256:], V[:, :, 256:], Kn, Vn)
        rows = [torch.cat([b, t[:, :, 256:].float()], 2) for b, t in zip(lagkv.dequantize(x, FL), (K, V))]
        near = lagkv.attend(q.float(), rows[0], rows[1], Kn.float(), Vn.float(), want_lse=True)
        bound = want[2] + A.attend(q.float(), rows[0], rows[1], Kn.float(), Vn.float())[2]
        assert bool(((got.out.double() - near.out.double()).abs().cpu() <= bound).all())
