"""Attention over a cache in 8 bits at the ends of its sizes: rows whose number nearly fills 31 bits, more than 2^24 query rows, outputs on the
queries."""
import math

import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv
from test_attend_quantized import BF, CODES, DEV, E4, FL, HF, I8, problem, rand, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 40], ids=["few_rows", "many_rows"])
def test_rows_that_nearly_fill_31_bits(N):
    """One row of codes, repeated (a row stride of 0): all weights are alike, and the outputs its values."""
    D, T = 16, 2 ** 31 - 2 ** 16 - 7
    one = torch.tensor([[[[(5 * i) % 23 - 11 for i in range(D)]]]], dtype=I8, device=DEV)
    scale = torch.full((1, 1, -(-T // 1024)), 0.125, device=DEV)
    q = rand(1, 2, N, D, dtype=BF, seed=1)
    lengths = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=DEV)
    x = lagkv.Quantized(one.expand(1, 1, T, D), one.expand(1, 1, T, D), scale, scale, 1024)
    got = lagkv.attend_quantized(q, x, lengths=lengths, want_lse=True)
    row = one[0, 0, 0].double().cpu() * 0.125
    # The sum is of 2^31 equal numbers, some 2^16 at a time in one register (each addition off by 2^-24 of what is there), the outputs' numerators likewise:
    # 2^17 * 2^-24 of each at most, and the output's rounding.
    assert bool((got.out.double().cpu() - row).abs().max() <= (2.0 ** -8 + 2 * 2.0 ** -7) * row.abs().max())
    want = (q.double().cpu() @ row) / math.sqrt(D) + math.log(T)
    assert bool((got.lse.double().cpu() - want).abs().max() <= 2.0 ** -7 + 1e-4)


def test_more_than_2_to_the_24_query_rows():
    G, N, D, T = 4, 2 ** 22 + 5, 16, 40
    q = rand(1, N, G, D, dtype=BF, seed=2).transpose(1, 2)
    x = stored(1, 1, T, D, 16, E4, 3)
    got = lagkv.attend_quantized(q, x, want_lse=True)
    for at in (0, 1, 2 ** 21, 2 ** 22 - 3, N - 4):
        pick = slice(at, at + 4)
        A.check(lagkv.Attended(got.out[:, :, pick], got.lse[:, :, pick]), Q.attend(q[:, :, pick], x), str(at))


@CODES
@pytest.mark.parametrize("dtype,N", [(BF, 1), (BF, 70), (HF, 70), (FL, 20)], ids=["bf16-1", "bf16-70", "f16-70", "f32-20"])
def test_outputs_on_the_queries(dtype, N, code):
    q, x, *rows = problem(dtype, code, 2, 2, 4, N, 128, 700, 60, "chain", 32, seed=6)
    want = lagkv.attend_quantized(q, x, *rows, want_lse=True)
    same = q.clone(memory_format=torch.preserve_format)
    got = lagkv.attend_quantized(same, x, *rows, out=same, want_lse=True)
    assert got.out is same and torch.equal(same, want.out) and torch.equal(got.lse, want.lse)


@CODES
@pytest.mark.parametrize("dtype,N", [(BF, 1), (BF, 70), (HF, 70), (FL, 3)], ids=["bf16-1", "bf16-70", "f16-70", "f32-3"])
def test_scales_at_the_end_of_the_range(dtype, N, code):
    """Scales of V from the smallest number to 2^118, at which the weighted sums of 300 rows are still numbers."""
    q, x, Kt, Vt, Kn, Vn = problem(dtype, code, 1, 2, 2, N, 64, 300, 10, "chain", 16, seed=7)
    small = torch.randint(0, 2, x.V.shape, generator=torch.Generator().manual_seed(1), dtype=I8).to(DEV)
    x.V.view(I8).copy_(small)                  # (0 and 1, or 0 and 2^-9)
    x.V_scale.fill_(2.0 ** 118 if dtype != HF else 2.0 ** 15)
    A.check(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True), Q.attend(q, x, Kt, Vt, Kn, Vn))
    x.V_scale[:, :, ::2] = 2.0 ** -149
    A.check(lagkv.attend_quantized(q, x, Kt, Vt, Kn, Vn, want_lse=True), Q.attend(q, x, Kt, Vt, Kn, Vn))
