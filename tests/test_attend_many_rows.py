"""The kernel of many query rows in every form that a call can reach: tiles of 128 and 256 rows, one piece of the cache and several,
each named by lagkv_attend_plan, at the lengths, trees, values and scales where they can go wrong.  (The eight wavefronts of a
256-row tile go in two halves a phase apart.)"""
import math

import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv
from test_attend_infinite import CODE, rand, same

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16
TYPES = pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])


def plan_is(dtype, B, G, N, D, T, tile, pieces):
    x = lagkv.attend_plan(lagkv.AttendParams(B, 1, G, N, D, CODE[dtype], 0, 0, T, 0.1))
    assert (x.many_rows, x.row_tile, x.wavefronts) == (1, tile, tile // 32) and (x.pieces > 1) == (pieces > 1), (x.row_tile, x.pieces)


def problem(dtype, B, G, N, D, T, seed):
    q = rand(B, N, G, D, dtype=dtype, seed=seed).transpose(1, 2)
    return q, *(rand(B, 1, n, D, dtype=dtype, seed=seed + 1 + i) for i, n in enumerate((T, T, N, N)))


def tree(N, seed, B=1, padded=0):
    g = torch.Generator().manual_seed(seed)
    p = torch.tensor([[int(torch.randint(max(-1, n - 6), n, (1,), generator=g)) for n in range(N)] for _ in range(B)], dtype=torch.int32)
    for i in range(padded):
        p[:, N - 1 - 3 * i] = -2 if i % 2 == 0 else 1000
    return p.to(DEV)


def of_copies(copies, args, parents, **kw):
    got = lagkv.attend(*(t.expand(copies, *t.shape[1:]) for t in args), parents, want_lse=True, **kw)
    assert bool((got.out.nan_to_num(7.0) == got.out[:1].nan_to_num(7.0)).all()) and bool((got.lse.nan_to_num(7.0) == got.lse[:1].nan_to_num(7.0)).all())
    return lagkv.Attended(got.out[:1], got.lse[:1])


FORMS = [  # streams, G, N, D, T, rows of a tile, pieces
    (1200, 4, 20, 64, 200, 128, 1), (1200, 4, 33, 48, 90, 128, 1), (8, 4, 64, 64, 4000, 128, 2), (1200, 2, 60, 100, 130, 128, 1),
    (4, 4, 64, 128, 4000, 128, 2), (1200, 4, 10, 256, 90, 128, 1), (8, 4, 30, 200, 3000, 128, 2),
    (200, 4, 40, 128, 200, 256, 1), (200, 1, 256, 72, 200, 256, 1), (100, 2, 130, 100, 700, 256, 1), (64, 4, 40, 128, 1500, 256, 2),
    (64, 2, 130, 80, 700, 256, 2), (40, 2, 130, 128, 1500, 256, 2), (200, 5, 50, 121, 700, 256, 1),
]


@TYPES
@pytest.mark.parametrize("new", ["chain", "tree"])
@pytest.mark.parametrize("form", FORMS, ids=lambda s: "x".join(map(str, s)))
def test_forms(form, new, dtype):
    copies, G, N, D, T, tile, pieces = form
    print("[gpu-test] many rows", form, new, dtype, flush=True)
    plan_is(dtype, copies, G, N, D, T, tile, pieces)
    args = problem(dtype, 1, G, N, D, T, D + T)
    parents = tree(N, T)[0] if new == "tree" else None
    A.check(of_copies(copies, args, parents), A.attend(*args, parents), str(form))


@TYPES
@pytest.mark.parametrize("new", ["none", "chain", "tree"])
@pytest.mark.parametrize("form", [(200, 4, 40, 128, 200, 256, 1), (64, 4, 40, 100, 1500, 256, 2), (1200, 4, 20, 64, 200, 128, 1), (64, 4, 20, 64, 4000, 128, 2)],
                         ids=lambda s: "x".join(map(str, s)))
def test_ragged_lengths_and_padded_trees(form, new, dtype):
    """What lies behind a length, and the rows of what is no token, is NaN and infinite."""
    copies, G, N, D, T, tile, pieces = form
    plan_is(dtype, copies, G, N, D, T, tile, pieces)
    lens = [0, 1, 64, 65, 127, T, 5 * T, -7] if pieces == 1 else [0, 1, T // 2, T - 1]
    n = len(lens)
    q, K, V, Kn, Vn = problem(dtype, n, G, N, D, T, 3)
    parents = tree(N, 1, n, padded=3) if new == "tree" else None
    if new == "none":
        Kn = Vn = None
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = A.attend(q, K, V, Kn, Vn, parents, lengths)
    for b, rows in enumerate(lens):
        rows = min(max(rows, 0), T)
        K[b, :, rows:], V[b, :, rows:] = math.nan, math.inf
    if parents is not None:
        none = (parents < -1) | (parents >= torch.arange(N, device=DEV))
        assert int(none.sum()) == 3 * n
        Kn.transpose(1, 2)[none], Vn.transpose(1, 2)[none] = math.nan, -math.inf
    r = lambda t: None if t is None else t.repeat(copies // n, *[1] * (t.dim() - 1))
    got = lagkv.attend(r(q), r(K), r(V), r(Kn), r(Vn), r(parents), r(lengths), want_lse=True)
    A.check(lagkv.Attended(got.out[:n], got.lse[:n]), want, str(form))
    assert torch.equal(got.out, r(got.out[:n])) and torch.equal(got.lse, r(got.lse[:n]))


ODD = [(200, 1, 256, 128, 200, 256, 1), (100, 2, 130, 100, 700, 256, 1), (40, 2, 130, 128, 1500, 256, 2), (1200, 2, 70, 64, 90, 128, 1),
       (4, 2, 200, 128, 4000, 128, 2), (1200, 1, 130, 256, 90, 128, 1)]


@TYPES
@pytest.mark.parametrize("chain", [True, False], ids=["chain", "tree"])
@pytest.mark.parametrize("form", ODD, ids=lambda s: "x".join(map(str, s)))
def test_infinite_rows_of_new_tokens(form, chain, dtype):
    """Values of tokens in several steps, some infinite, some none; a key of one: they reach the tokens that see them, and no others."""
    copies, G, N, D, T, tile, pieces = form
    plan_is(dtype, copies, G, N, D, T, tile, pieces)
    args = q, K, V, Kn, Vn = problem(dtype, 1, G, N, D, T, 9)
    parents = None if chain else tree(N, 5)[0]
    at = [3, N // 4, N // 2, N - 2]
    Vn[0, 0, at[0], 7], Vn[0, 0, at[1], D - 1], Vn[0, 0, at[2], 8], Vn[0, 0, at[3], 7] = math.inf, -math.inf, math.nan, -math.inf
    V[0, 0, T // 2, 11] = math.inf
    want = A.attend(*args, parents)
    odd = ~torch.isfinite(want[0][0, 0])
    assert all(bool(odd[:, c].any()) for c in (7, D - 1, 8)) and not bool(odd[:, 7].all()) and bool(odd[:, 11].all())
    same(of_copies(copies, args, parents), want, "values")
    Kn[0, 0, at[2], 5], K[0, 0, T - 1, 0] = math.nan, 0.0
    q[0, 0, N // 3, 2] = math.nan
    same(of_copies(copies, args, parents), A.attend(*args, parents), "keys")


@TYPES
@pytest.mark.parametrize("form", [(200, 4, 40, 128, 200, 256, 1), (64, 4, 40, 100, 1500, 256, 2), (1200, 4, 20, 64, 200, 128, 1), (4, 4, 64, 128, 4000, 128, 2),
                                  (1200, 4, 10, 256, 90, 128, 1)], ids=lambda s: "x".join(map(str, s)))
def test_scales(form, dtype):
    copies, G, N, D, T, tile, pieces = form
    plan_is(dtype, copies, G, N, D, T, tile, pieces)
    args = problem(dtype, 1, G, N, D, T, 21)
    parents = tree(N, 2)[0]
    for scale in (-0.2, 0.0, 1.5, 1e-40):
        A.check(of_copies(copies, args, parents, scale=scale), A.attend(*args, parents, scale=scale), str(scale))


@TYPES
@pytest.mark.parametrize("form", [(200, 4, 40, 128, 200, 256, 1), (64, 4, 40, 100, 1500, 256, 2), (1200, 4, 20, 64, 200, 128, 1)], ids=lambda s: "x".join(map(str, s)))
def test_the_output_in_place_of_the_queries_and_one_layer_of_a_cache(form, dtype):
    copies, G, N, D, T, tile, pieces = form
    plan_is(dtype, copies, G, N, D, T, tile, pieces)
    q, K, V, Kn, Vn = args = problem(dtype, 1, G, N, D, T, 46)
    want = A.attend(*args)
    room = torch.full((2, 1, 1, T + 9, D + 5), math.nan, dtype=dtype, device=DEV)
    room[0, ..., :T, 1:D + 1], room[1, ..., :T, 1:D + 1] = K, V
    big = q.repeat(copies, 1, 1, 1)
    got = lagkv.attend(big, *(room[i, ..., :T, 1:D + 1].expand(copies, 1, T, D) for i in range(2)), *(t.expand(copies, 1, N, D) for t in (Kn, Vn)), out=big, want_lse=True)
    assert got.out is big and bool((big == big[:1]).all())
    A.check(lagkv.Attended(big[:1], got.lse[:1]), want)
