"""Rows into 8-bit codes with a scale for each block, and back, against plain 64-bit forms: codes have to be equal."""
import math

import pytest
import torch

import quant_util as Q
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn
MARK = 85


def rows(B, H, T, D, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, H, T, D), generator=g) * torch.exp(torch.randn((B, H, T, 1), generator=g)) * scale
    return x.to(dtype).to(DEV)


def room(B, H, T, D, block, code):
    """Codes and scales that are marked, to see what is written."""
    x = lagkv.Quantized.empty(B, H, T, D, block, code, DEV)
    for t in (x.K, x.V):
        t.view(torch.int8).fill_(MARK)
    for t in (x.K_scale, x.V_scale):
        t.fill_(-3.0)
    return x


def check(x, K, V, block, code, lengths=None, start=0):
    first = start // block * block if start < K.shape[2] else K.shape[2]
    for codes, scale, rows_ in ((x.K, x.K_scale, K), (x.V, x.V_scale, V)):
        want, want_scale, written = Q.quantize(rows_, block, code, lengths)
        written[:, :, :first] = False
        got, got_scale = codes.cpu(), scale.cpu()
        raw = got.view(torch.int8)
        assert bool((raw[~written] == MARK).all()), "rows that are not there were written"
        assert torch.equal(got.float().to(Q.F64)[written], want[written] + 0.0), \
            f"codes differ: {int((got.float().to(Q.F64)[written] != want[written]).sum())} of {int(written.sum()) * want.shape[3]}"
        blocks = written[:, :, ::block]
        assert bool((got_scale[~blocks] == -3.0).all())
        assert torch.equal(torch.isnan(got_scale[blocks]), torch.isnan(want_scale[blocks]))
        fine = blocks & torch.isfinite(want_scale)
        assert torch.equal(got_scale[fine].to(Q.F64), want_scale[fine])


SIZES = [  # B, H, T, D, block
    (1, 1, 1, 16, 16), (1, 2, 17, 64, 16), (2, 3, 100, 128, 32), (1, 2, 130, 128, 64), (2, 1, 200, 80, 64),
    (1, 1, 300, 100, 128), (1, 2, 77, 41, 16), (1, 1, 260, 250, 128), (1, 1, 700, 256, 512), (1, 1, 1500, 17, 1024),
    (3, 2, 65, 96, 64), (1, 1, 1030, 128, 1024),
]


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_rows_into_codes_and_back(size, dtype, code):
    B, H, T, D, block = size
    print("[gpu-test] quantize", size, dtype, code, flush=True)
    K, V = rows(B, H, T, D, dtype, 1), rows(B, H, T, D, dtype, 2)
    x = room(B, H, T, D, block, code)
    assert lagkv.quantize(K, V, block, out=x) is x
    check(x, K, V, block, code)
    for to in (BF, HF, FL):
        for got, codes, scale in zip(lagkv.dequantize(x, to), (x.K, x.V), (x.K_scale, x.V_scale)):
            # code * scale rounded to fp32, then to the type: as torch does it
            each = scale.repeat_interleave(block, 2)[:, :, :T, None]
            assert torch.equal(got, (codes.float() * each).to(to))


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
def test_ties_and_their_neighbours(dtype, code):
    """Blocks of every quotient (k + 1/2) / 127 that the type holds, of its neighbours, and of all magnitudes of maxima."""
    block, D = 16, 64
    g = torch.Generator().manual_seed(5)
    tops = torch.cat([torch.tensor([1.0, 2.0, 127.0, 254.0, 0.5, 3.0, 1.984375, 448.0, 449.0, 1.75, 1.7578125, 896.0]),
                      1 + torch.randint(0, 128, (20,), generator=g) / 128.0])
    K = torch.zeros(1, len(tops), block, D, dtype=FL)
    for i, a in enumerate(tops.tolist()):
        k = torch.randint(0, 127, (block, D), generator=g) + 0.5
        x = (k * a / 127).to(dtype).to(FL)
        if code == E4:
            x = torch.randint(0, 4096, (block, D), generator=g) * a / 4096
        if dtype == FL:  # one step to either side
            x = torch.nextafter(x, torch.where(torch.rand(x.shape, generator=g) < 0.5, math.inf, -math.inf))
        x[::2] *= -1
        x[3, 5] = a
        K[0, i] = x.clamp(-a, a)
    K = K.to(dtype).to(DEV)
    V = (K.float() * torch.exp2(torch.arange(len(tops), device=DEV).float() % 7 - 3)[None, :, None, None]).to(dtype)
    x = room(1, len(tops), block, D, block, code)
    lagkv.quantize(K, V, block, out=x)
    check(x, K, V, block, code)


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
def test_values_at_the_ends_of_the_range(code):
    tops = [0.0, 2.0 ** -149, 2.0 ** -140, 3e-39, 1.2e-38, 1e-30, 1e-19, 2.0 ** 63, 2.0 ** 64, 1e30, 3.4028234e38]
    g = torch.Generator().manual_seed(6)
    K = (torch.rand(1, len(tops), 32, 32, generator=g, dtype=torch.float64) * 2 - 1) * torch.tensor(tops, dtype=torch.float64)[None, :, None, None]
    K[0, :, 0, 0] = torch.tensor(tops, dtype=torch.float64)
    for dtype in (FL, BF):
        k = K.to(dtype).nan_to_num(posinf=3e38, neginf=-3e38).to(DEV)
        x = room(1, len(tops), 32, 32, 32, code)
        lagkv.quantize(k, -k, 32, out=x)
        check(x, k, -k, 32, code)


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
def test_what_is_no_number(dtype, code):
    """A block with an infinity or NaN: all of it reads back as NaN, and no other one."""
    K, V = rows(1, 1, 96, 48, dtype, 3), rows(1, 1, 96, 48, dtype, 4)
    K[0, 0, 40, 47], V[0, 0, 0, 0], V[0, 0, 95, 1] = math.nan, math.inf, -math.inf
    x = room(1, 1, 96, 48, 32, code)
    lagkv.quantize(K, V, 32, out=x)
    check(x, K, V, 32, code)
    k, v = lagkv.dequantize(x, dtype)
    assert bool(torch.isnan(k[0, 0, 32:64]).all()) and bool(torch.isfinite(k[0, 0, :32]).all()) and bool(torch.isfinite(k[0, 0, 64:]).all())
    assert bool(torch.isnan(v[0, 0, :32]).all()) and bool(torch.isfinite(v[0, 0, 32:64]).all()) and bool(torch.isnan(v[0, 0, 64:]).all())


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 64, 256])
@pytest.mark.parametrize("start", [0, 1, 64, 100, 199, 200, 1000])
def test_lengths_and_starts(start, block, code):
    """Rows behind a length hold NaN and are neither read into a scale nor written; nor are blocks before `start`'s."""
    T, lens = 200, [0, 1, 64, 65, 130, 200, 999, -5]
    K, V = rows(len(lens), 2, T, 24, BF, 7), rows(len(lens), 2, T, 24, BF, 8)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        K[b, :, max(n, 0):], V[b, :, max(n, 0):] = math.nan, math.inf
    x = room(len(lens), 2, T, 24, block, code)
    lagkv.quantize(K, V, block, lengths=lengths, start=start, out=x)
    check(x, K, V, block, code, lengths, start)
    full = lagkv.quantize(K, V, block, code, lengths)
    out = tuple(torch.full_like(K, 7.0) for _ in range(2))
    assert lagkv.dequantize(full, lengths=lengths, start=start, out=out)[0] is out[0]
    for got, codes, scale in zip(out, (full.K, full.V), (full.K_scale, full.V_scale)):
        want = (codes.float() * scale.repeat_interleave(block, 2)[:, :, :T, None]).to(BF)
        for b, n in enumerate(lens):
            n = min(max(n, start), T)
            assert torch.equal(got[b, :, start:n], want[b, :, start:n])
            assert bool((got[b, :, n:] == 7.0).all()) and bool((got[b, :, :start] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
def test_strides(dtype):
    """Rows of a projection's output, codes in a larger store with padding between rows, odd addresses."""
    B, H, T, D, block = 2, 3, 70, 37, 32
    K, V = (rows(B, T, H, D + 3, dtype, i)[..., 1:1 + D].transpose(1, 2) for i in (9, 10))
    store = torch.full((2, B, 80, H, D + 5), MARK, dtype=torch.int8, device=DEV)
    scales = torch.full((2, B, H, 9), -3.0, device=DEV)
    x = lagkv.Quantized(*(store[i, :, 3:3 + T, :, 2:2 + D].transpose(1, 2) for i in range(2)), *(scales[i, :, :, 1:4] for i in range(2)), block)
    lagkv.quantize(K, V, block, out=x)
    check(x, K, V, block, I8)
    inside = torch.zeros_like(store, dtype=torch.bool)
    inside[:, :, 3:3 + T, :, 2:2 + D] = True
    assert bool((store[~inside] == MARK).all()) and bool((scales[..., 0] == -3.0).all()) and bool((scales[..., 4:] == -3.0).all())
    out = torch.full((2, B, T, H, D + 1), 7.0, dtype=dtype, device=DEV)
    k, v = lagkv.dequantize(x, out=tuple(out[i, ..., 1:].transpose(1, 2) for i in range(2)))
    assert torch.equal(k, (x.K.float() * x.K_scale.repeat_interleave(block, 2)[:, :, :T, None]).to(dtype))
    assert torch.equal(v, (x.V.float() * x.V_scale.repeat_interleave(block, 2)[:, :, :T, None]).to(dtype)) and bool((out[..., 0] == 7.0).all())


def test_one_head_for_all():
    """A stride of 0 repeats what is read."""
    K = rows(1, 1, 64, 32, BF, 11).expand(2, 4, 64, 32)
    x = lagkv.quantize(K, K, 16)
    assert x.K.shape == (2, 4, 64, 32) and torch.equal(x.K[1, 3], x.K[0, 0])
    shared = lagkv.Quantized(x.K[:1, :1].expand(2, 4, 64, 32), x.V[:1, :1].expand(2, 4, 64, 32), x.K_scale[:1, :1].expand(2, 4, 4),
                             x.V_scale[:1, :1].expand(2, 4, 4), 16)
    assert torch.equal(lagkv.dequantize(shared)[0], lagkv.dequantize(x)[0])


def test_an_update_gives_what_the_whole_gives():
    K, V = rows(2, 2, 300, 64, BF, 12), rows(2, 2, 300, 64, BF, 13)
    x = lagkv.Quantized.empty(2, 2, 320, 64, 64, I8, DEV)
    done = 0
    for n in (1, 63, 64, 65, 200, 300):
        lagkv.quantize(K[:, :, :n], V[:, :, :n], 64, start=done, out=x.view(n))
        done = n
    want = lagkv.quantize(K, V, 64)
    got = x.view(300)
    for a, b in zip((got.K, got.V, got.K_scale, got.V_scale), (want.K, want.V, want.K_scale, want.V_scale)):
        assert torch.equal(a, b)


def test_no_rows():
    x = lagkv.quantize(*(torch.empty(1, 2, 0, 64, dtype=BF, device=DEV) for _ in range(2)), 16)
    assert x.K.shape == (1, 2, 0, 64) and x.K_scale.shape == (1, 2, 0)
    assert lagkv.dequantize(x)[0].shape == (1, 2, 0, 64)


@pytest.mark.parametrize("code", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype,D,block", [(BF, 128, 64), (HF, 100, 32), (FL, 96, 128), (BF, 256, 256), (FL, 17, 16)], ids=lambda v: str(v).split(".")[-1])
def test_more_rows_than_the_caches_hold(dtype, D, block, code):
    """Copies of a cache (a batch stride of 0), together more than 256 MB: the codes of each are those of one, and rows behind a length are left."""
    T, B = 5000 + block // 2, 1 + 280_000_000 // (2 * 5000 * D * (4 if dtype == FL else 2))
    g = torch.Generator().manual_seed(D)
    K, V = (torch.randn((1, 1, T, D), generator=g).to(dtype).to(DEV) for _ in range(2))
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    lengths[1::2] = 777
    out = lagkv.Quantized.empty(B, 1, T, D, block, code)
    for t in (out.K, out.V):
        t.view(torch.int8).fill_(85)
    got = lagkv.quantize(K.expand(B, 1, T, D), V.expand(B, 1, T, D), block, code, lengths, out=out)
    for b in range(2):
        n = int(lengths[b])
        one = lagkv.quantize(K[:, :, :n], V[:, :, :n], block, code)
        for big, small in ((got.K, one.K), (got.V, one.V)):
            big, small = big.view(torch.int8)[b::2], small.view(torch.int8)
            assert bool((big[:, :, :n] == small).all()) and bool((big[:, :, n:] == 85).all())
        for big, small in ((got.K_scale, one.K_scale), (got.V_scale, one.V_scale)):
            assert bool((big[b::2, :, :-(-n // block)] == small).all())
