"""Attention over a cache in 8 bits where the largest scales of V are of rows that no token sees much of: what the others give must not be lost
against them."""
import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv
from test_attend_quantized import BF, CODES, FL, HF, TYPES, problem, tree
from test_attend_quantized_many_rows import of_many

pytestmark = pytest.mark.gpu


def without(x, far):
    """x without the blocks that `far` lists."""
    block, nb = x.block, x.K_scale.shape[2]
    rows = torch.tensor([r for r in range(x.K.shape[2]) if r // block not in far], device=x.K.device)
    blocks = torch.tensor([j for j in range(nb) if j not in far], device=x.K.device)
    take = lambda t: t.view(torch.int8)[:, :, rows].view(t.dtype)  # noqa: E731
    return lagkv.Quantized(take(x.K), take(x.V), x.K_scale[:, :, blocks].contiguous(), x.V_scale[:, :, blocks].contiguous(), block)


def unseen(q, x, far, ratio):
    """Makes the blocks `far` ones of logits below -900 in channel 0 alone, and of scales of V `ratio` times the others' largest."""
    q[..., 0] = 8.0
    D, block, most = q.shape[3], x.block, x.V_scale.max()
    for j in far:
        at = slice(j * block, (j + 1) * block)
        x.K.view(torch.int8)[:, :, at] = 0
        x.K[:, :, at, 0] = torch.tensor(-120.0).to(x.K.dtype)
        x.K_scale[:, :, j] = 1.0 * D ** 0.5  # (8 * -120 * D^0.5 / D^0.5: a weight of e^-900, which is 0 beside any other)
        x.V_scale[:, :, j] = most * ratio


RATIOS = pytest.mark.parametrize("ratio", [2.0 ** 9, 2.0 ** 20, 2.0 ** 70], ids=["2^9", "2^20", "2^70"])
FAR = pytest.mark.parametrize("far", [(0,), (4,), (9,), (0, 3, 8)], ids=str)


@CODES
@TYPES
@RATIOS
@FAR
@pytest.mark.parametrize("G,N,D", [(1, 1, 128), (4, 7, 64), (2, 3, 250)])
def test_few_rows(G, N, D, far, ratio, dtype, code):
    q, x, *rows = problem(dtype, code, 1, 2, G, N, D, 16 * 10, 0, "none", 16, seed=D + N)
    unseen(q, x, far, ratio)
    got = lagkv.attend_quantized(q, x, *rows, want_lse=True)
    A.check(got, Q.attend(q, without(x, far), *rows), f"{far} {ratio}")


@CODES
@TYPES
def test_the_largest_ratio(dtype, code):
    """Scales of V 2^100 apart (what goes by the query rows has no limit but fp32's)."""
    q, x, *rows = problem(dtype, code, 2, 1, 4, 2, 128, 16 * 40, 20, "chain", 16, seed=5)
    x.V_scale.mul_(2.0 ** -10)
    if dtype == HF:
        x.V_scale.mul_(2.0 ** 10)
    far = (0, 1, 17, 38)
    unseen(q, x, far, 2.0 ** 100)
    got = lagkv.attend_quantized(q, x, *rows, want_lse=True)
    A.check(got, Q.attend(q, without(x, far), *rows), "2^100")


@CODES
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@RATIOS
@FAR
@pytest.mark.parametrize("G,N,D,new", [(3, 50, 128, "chain"), (4, 20, 64, "tree"), (2, 65, 256, "none")])
def test_many_rows(G, N, D, new, far, ratio, dtype, code):
    q, x, *rows = problem(dtype, code, 1, 1, G, N, D, 64 * 10, 20, new, 64, seed=D + N)
    unseen(q, x, far, ratio)
    parents = tree(N, 3) if new == "tree" else None
    got = of_many(q, x, *rows, parents)
    A.check(got, Q.attend(q, without(x, far), *rows, parents), f"{far} {ratio}")


@CODES
@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
def test_some_tokens_see_them(dtype, code):
    """Of two tokens one sees nothing of the rows of large scales, the other little else."""
    q, x, *rows = problem(dtype, code, 1, 1, 1, 2, 128, 16 * 10, 0, "none", 16, seed=8)
    far = (2, 7)
    unseen(q, x, far, 2.0 ** 20)
    q[:, :, 1, 0] = -8.0
    got = lagkv.attend_quantized(q, x, *rows, want_lse=True)
    first, second = (lagkv.Attended(got.out[:, :, n:n + 1], got.lse[:, :, n:n + 1]) for n in range(2))
    A.check(first, Q.attend(q[:, :, :1], without(x, far), *rows), "unseen")
    A.check(second, Q.attend(q[:, :, 1:], x, *rows), "seen")
