"""The operators that read a cache against plain 64-bit forms: attention of new tokens, bounds of blocks, the selection of
blocks and attention over them, at the sizes, strides, masks and values where they can go wrong."""
import math

import pytest
import torch

import attend_util as A
from paper_2504_04704_amd import lagkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def rand(*shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def problem(dtype, B, H, G, N, D, T, new, seed=0):
    """q, K, V, K_new, V_new; a few strong channels, so that the softmax is neither flat nor a single row."""
    q = rand(B, N, H * G, D, dtype=dtype, seed=seed).transpose(1, 2)
    K, V = rand(B, H, T, D, dtype=dtype, seed=seed + 1, scale=1.5), rand(B, H, T, D, dtype=dtype, seed=seed + 2)
    if new == "none":
        return q, K, V, None, None
    return q, K, V, rand(B, H, N, D, dtype=dtype, seed=seed + 3), rand(B, H, N, D, dtype=dtype, seed=seed + 4)


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


SIZES = [  # B, H, G, N, D, T, new
    (1, 1, 1, 1, 64, 1, "none"),
    (1, 2, 2, 1, 64, 0, "chain"),
    (2, 1, 3, 1, 128, 31, "chain"),
    (1, 2, 4, 1, 128, 33, "chain"),
    (2, 2, 8, 1, 80, 257, "none"),
    (1, 1, 5, 7, 96, 130, "tree"),
    (2, 2, 4, 8, 128, 515, "tree"),       # 32 query rows: one tile
    (1, 2, 4, 9, 128, 300, "tree"),       # 36: two
    (1, 1, 2, 33, 64, 65, "tree"),
    (1, 1, 1, 70, 128, 20, "tree"),       # three words of ancestors
    (1, 1, 3, 50, 128, 100, "chain"),
    (1, 1, 2, 1, 256, 100, "chain"),
    (1, 2, 3, 5, 256, 77, "tree"),
    (1, 1, 2, 3, 8, 50, "chain"),         # the narrowest head
    (1, 2, 2, 2, 41, 90, "tree"),         # rows on odd addresses
    (1, 1, 4, 2, 100, 70, "tree"),
    (1, 1, 6, 3, 250, 40, "chain"),
    (1, 1, 1, 1, 128, 3000, "chain"),     # the cache in pieces
    (1, 1, 4, 16, 128, 2500, "tree"),
    (2, 1, 130, 1, 64, 90, "chain"),      # more query heads than a tile
    (1, 2, 4, 40, 128, 700, "tree"),      # many query rows: 160, of 256
    (1, 1, 5, 60, 128, 190, "chain"),     # 300: two tiles
    (1, 1, 2, 130, 64, 129, "chain"),
    (1, 1, 3, 12, 41, 100, "tree"),       # rows on odd addresses
    (1, 2, 7, 21, 100, 230, "chain"),
    (1, 1, 4, 20, 250, 150, "tree"),
    (1, 1, 2, 65, 256, 60, "chain"),
    (1, 1, 8, 16, 128, 3000, "tree"),     # the cache in pieces
    (1, 1, 1, 256, 64, 10, "tree"),       # the largest tree
    (1, 2, 8, 6, 96, 0, "tree"),
]


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_attend(size, dtype):
    B, H, G, N, D, T, new = size
    print("[gpu-test] attend", size, dtype, flush=True)
    q, K, V, Kn, Vn = problem(dtype, B, H, G, N, D, T, new, seed=D + T)
    parents = tree(N, T, B) if new == "tree" else None
    got = lagkv.attend(q, K, V, Kn, Vn, parents, want_lse=True)
    assert got.out.stride() == q.stride()
    A.check(got, A.attend(q, K, V, Kn, Vn, parents), str(size))


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", ["none", "chain", "tree"])
@pytest.mark.parametrize("N", [5, 20])
def test_ragged_lengths_and_what_lies_behind_them(dtype, new, N):
    """Lengths of nothing, of one row, inside and at the end of a step, and beyond the rows there are; the rows behind
    them, which a cache has not written yet, hold NaN and infinities."""
    T = 200
    lens = [0, 1, 16, 33, 100, 200, 1000, -7]
    q, K, V, Kn, Vn = problem(dtype, len(lens), 2, 4, N, 64, T, new, seed=3)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    parents = tree(N, 1) if new == "tree" else None
    clean = A.attend(q, K, V, Kn, Vn, parents, lengths)
    for b, n in enumerate(lens):
        n = min(max(n, 0), T)
        K[b, :, n:], V[b, :, n:] = math.nan, math.inf
    got = lagkv.attend(q, K, V, Kn, Vn, parents, lengths, want_lse=True)
    A.check(got, clean)
    if new == "none":
        assert bool((got.out[0] == 0).all()) and bool((got.lse[7] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 12], ids=["few_rows", "many_rows"])
def test_ragged_lengths_of_a_cache_in_pieces(dtype, N):
    """Pieces that are cut for the longest length there may be: most have no row of a shorter one."""
    T, lens = 5000, [0, 1, 70, 4999]
    q, K, V, Kn, Vn = problem(dtype, len(lens), 1, 4, N, 64, T, "chain", seed=15)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = A.attend(q, K, V, Kn, Vn, None, lengths)
    for b, n in enumerate(lens):
        K[b, :, n:], V[b, :, n:] = math.nan, math.nan
    A.check(lagkv.attend(q, K, V, Kn, Vn, lengths=lengths, want_lse=True), want)


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 1, 8, 1, 128, 60001), (1, 1, 4, 30, 64, 20000), (3, 5, 2, 1, 64, 5000), (1, 3, 4, 9, 128, 7000),
                                  (1, 7, 32, 1, 100, 3001), (1, 1, 2, 17, 256, 9000)], ids=lambda s: "x".join(map(str, s)))
def test_many_pieces_of_few_streams(dtype, size):
    """Caches that are cut into numbers of pieces that are no multiples of the eight chiplets', of one stream and more."""
    B, H, G, N, D, T = size
    q, K, V, Kn, Vn = problem(dtype, B, H, G, N, D, T, "chain", seed=T)
    A.check(lagkv.attend(q, K, V, Kn, Vn, want_lse=True), A.attend(q, K, V, Kn, Vn))


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("chain", [True, False])
def test_values_of_tokens_that_are_not_seen(dtype, bad, chain):
    """An infinite or undefined row of a new token reaches those that see it, and no others."""
    N, T, at = 40, 50, 20
    q, K, V, Kn, Vn = problem(dtype, 1, 1, 2, N, 64, T, "tree", seed=9)
    parents = None if chain else tree(N, 5)
    want = A.attend(q, K, V, Kn, Vn, parents)
    see = A.tree_visible(parents.cpu(), N)[:, at] if not chain else torch.arange(N) >= at
    assert bool(see.any()) and bool((~see).any())
    Vn[0, 0, at, 7] = bad
    got = lagkv.attend(q, K, V, Kn, Vn, parents)
    assert not bool(torch.isfinite(got.out[0, :, see, 7]).any())
    keep = got.out.clone()
    keep[0, :, see] = want[0][0, :, see].to(dtype).to(DEV)
    A.check(lagkv.Attended(keep, None), want)
    Kn[0, 0, at] = bad
    got = lagkv.attend(q, K, V, Kn, Vn, parents)
    keep = got.out.clone()
    keep[0, :, see] = want[0][0, :, see].to(dtype).to(DEV)
    A.check(lagkv.Attended(keep, None), want)


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("N,T", [(1, 32), (1, 0), (1, 3000), (24, 64), (24, 3000)])
def test_what_is_no_number_and_is_seen(dtype, N, T):
    """A query row, or the row of a token that sees little else, with NaN: its outputs are NaN, and no others."""
    q, K, V, Kn, Vn = problem(dtype, 1, 2, 3, N, 128, T, "chain", seed=31)
    want = A.attend(q, K, V, Kn, Vn)

    def nan_in(got, bad):
        assert bool(torch.isnan(got.out[0, bad]).all()) and bool(torch.isnan(got.lse[0, bad]).all())
        got.out[0, bad], got.lse[0, bad] = want[0][0, bad].to(dtype).to(DEV), want[1][0, bad].float().to(DEV)
        A.check(got, want)

    q2 = q.clone()
    q2[0, 4, N - 1, 5] = math.nan
    got = lagkv.attend(q2, K, V, Kn, Vn, want_lse=True)
    bad = torch.zeros(6, N, dtype=torch.bool)
    bad[4, N - 1] = True
    nan_in(got, bad)
    Kn[0, 1, N - 1, 9] = math.nan
    got = lagkv.attend(q, K, V, Kn, Vn, want_lse=True)
    bad[3:, N - 1] = True
    nan_in(got, bad)
    if T > 32:
        K[0, 0, :, 3] = math.nan
        got = lagkv.attend(q, K, V, Kn, Vn, want_lse=True)
        assert bool(torch.isnan(got.out[0, :3]).all()) and bool(torch.isnan(got.lse[0, :3]).all())
        lo, hi = lagkv.block_bounds(K, 16)
        blocks = lagkv.select_blocks(q, lo, hi, T, 16, 4, 1, 1)
        got = lagkv.attend_blocks(q, K, V, blocks, 16, want_lse=True)
        assert bool(torch.isnan(got.out[0, :3]).all()) and bool(torch.isfinite(got.out[0, 3:]).all())


# Tiles of many rows are taken where there is much to multiply: the same shapes, of many streams.  (One problem, read by all: its
# strides along the batch are 0.)
MANY = 1200


def copies(*tensors):
    return [None if t is None else t[:1].expand(MANY, *t.shape[1:]) for t in tensors]


def the_first_of(got):
    """The first copy's result; that of all the others is the same, bit for bit."""
    same = got.out.nan_to_num(7.0) == got.out[:1].nan_to_num(7.0)
    assert bool(same.all())
    if got.lse is not None:
        assert bool((got.lse.nan_to_num(7.0) == got.lse[:1].nan_to_num(7.0)).all())
    return lagkv.Attended(got.out[:1].clone(), None if got.lse is None else got.lse[:1].clone())


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("size", [s for s in SIZES if s[2] * s[3] > 32 and s[1] * s[2] * s[3] <= 420 and s[3] > 1], ids=lambda s: "x".join(map(str, s)))
def test_attend_of_many_streams(size, dtype):
    _, H, G, N, D, T, new = size
    print("[gpu-test] attend, many streams", size, dtype, flush=True)
    q, K, V, Kn, Vn = problem(dtype, 1, H, G, N, D, T, new, seed=D + T)
    parents = tree(N, T) if new == "tree" else None
    got = lagkv.attend(*copies(q, K, V, Kn, Vn), parents, want_lse=True)
    A.check(the_first_of(got), A.attend(q, K, V, Kn, Vn, parents), str(size))


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("chain", [True, False])
def test_values_of_tokens_that_are_not_seen_of_many_streams(dtype, bad, chain):
    N, T, at = 70, 90, 40
    q, K, V, Kn, Vn = problem(dtype, 1, 1, 2, N, 128, T, "tree", seed=9)
    parents = None if chain else tree(N, 5)
    want = A.attend(q, K, V, Kn, Vn, parents)
    see = A.tree_visible(parents.cpu(), N)[:, at] if not chain else torch.arange(N) >= at
    assert bool(see.any()) and bool((~see).any())
    Vn[0, 0, at, 7] = bad
    for row in (None, Kn):
        if row is not None:
            row[0, 0, at] = bad
        got = the_first_of(lagkv.attend(*copies(q, K, V, Kn, Vn), parents))
        if row is None:
            assert not bool(torch.isfinite(got.out[0, :, see, 7]).any())
        got.out[0, :, see] = want[0][0, :, see].to(dtype).to(DEV)
        A.check(got, want)


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_what_is_no_number_and_is_seen_of_many_streams(dtype):
    N, T = 70, 64
    q, K, V, Kn, Vn = problem(dtype, 1, 1, 2, N, 128, T, "chain", seed=31)
    want = A.attend(q, K, V, Kn, Vn)
    for what in ("query", "key", "keys"):
        q2, Kn2, K2, bad = q.clone(), Kn.clone(), K.clone(), torch.zeros(2, N, dtype=torch.bool)
        if what == "query":
            q2[0, 1, 3, 5] = math.nan
            bad[1, 3] = True
        elif what == "key":
            Kn2[0, 0, N - 1, 9] = math.nan
            bad[:, N - 1] = True
        else:
            K2[0, 0, :, 3] = math.nan
            bad[:] = True
        got = the_first_of(lagkv.attend(*copies(q2, K2, V, Kn2, Vn), want_lse=True))
        assert bool(torch.isnan(got.out[0, bad]).all()) and bool(torch.isnan(got.lse[0, bad]).all())
        got.out[0, bad], got.lse[0, bad] = want[0][0, bad].to(dtype).to(DEV), want[1][0, bad].float().to(DEV)
        A.check(got, want)


@pytest.mark.parametrize("new", ["none", "chain", "tree"])
def test_ragged_lengths_of_many_streams(new):
    """Lengths as above, and trees of several sizes, 150 times each; what lies behind is NaN and infinite."""
    T, N = 200, 20
    lens = [0, 1, 64, 65, 127, 200, 1000, -7]
    q, K, V, Kn, Vn = problem(BF, len(lens), 2, 4, N, 64, T, new, seed=3)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    parents = tree(N, 1, len(lens), padded=3) if new == "tree" else None
    clean = A.attend(q, K, V, Kn, Vn, parents, lengths)
    for b, n in enumerate(lens):
        n = min(max(n, 0), T)
        K[b, :, n:], V[b, :, n:] = math.nan, math.inf
    r = lambda t: None if t is None else t.repeat(150, *[1] * (t.dim() - 1))
    got = lagkv.attend(r(q), r(K), r(V), r(Kn), r(Vn), r(parents), r(lengths), want_lse=True)
    A.check(lagkv.Attended(got.out[:8], got.lse[:8]), clean)
    assert torch.equal(got.out, r(got.out[:8])) and torch.equal(got.lse, r(got.lse[:8]))


@pytest.mark.parametrize("size", [(4, 8, 4, 64, 128, 2100, "tree"), (1, 8, 4, 150, 256, 2000, "chain"), (2, 4, 8, 200, 100, 3000, "chain")],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_rows_of_long_caches(size):
    B, H, G, N, D, T, new = size
    q, K, V, Kn, Vn = problem(BF, B, H, G, N, D, T, new, seed=D + T)
    parents = tree(N, T, B) if new == "tree" else None
    got = lagkv.attend(q, K, V, Kn, Vn, parents, want_lse=True)
    # (every few heads of every batch entry)
    heads = [0, H * G // 2, H * G - 1]
    for b in range(B):
        for i in heads:
            pick = lambda t, j: None if t is None else t[b:b + 1, j:j + 1]
            want = A.attend(pick(q, i), *(pick(t, i // G) for t in (K, V, Kn, Vn)), None if parents is None else parents[b:b + 1])
            A.check(lagkv.Attended(pick(got.out, i), pick(got.lse, i)), want, f"{b} {i}")


def test_padded_trees():
    """Trees of several sizes in one batch: what is no token sees nothing and is not seen, nor is what lies before it on a
    path, and its rows may hold anything."""
    N = 12
    q, K, V, Kn, Vn = problem(BF, 3, 2, 2, N, 128, 60, "tree", seed=4)
    parents = tree(N, 8, 3, padded=4)
    parents[1, 0] = -5                       # a root that is no token: the paths that lead to it end before it
    parents[2, 3] = 3                        # its own parent
    want = A.attend(q, K, V, Kn, Vn, parents)
    none = torch.zeros(3, N, dtype=torch.bool)
    for b in range(3):
        for n in range(N):
            none[b, n] = int(parents[b, n]) < -1 or int(parents[b, n]) >= n
    assert int(none.sum()) >= 12
    for b in range(3):
        for n in range(N):
            if none[b, n]:
                Kn[b, :, n], Vn[b, :, n] = math.nan, math.nan
    q = q.contiguous()
    for b in range(3):
        q[b, :, none[b].to(DEV)] = math.nan
    got = lagkv.attend(q, K, V, Kn, Vn, parents, want_lse=True)
    A.check(got, want)
    assert bool((got.out.transpose(1, 2)[none.to(DEV)] == 0).all())


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
def test_strides(dtype):
    """[B,T,H,D] tensors, one layer of a cache with room, a cache that all of a batch shares, rows apart and on odd
    addresses, and an output between rows that stay as they were."""
    B, H, G, N, D, T = 2, 3, 2, 4, 72, 90
    q, K, V, Kn, Vn = problem(dtype, B, H, G, N, D, T, "chain", seed=12)
    want = A.attend(q, K, V, Kn, Vn)
    swap = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    A.check(lagkv.attend(q.contiguous(), swap(K), swap(V), swap(Kn), swap(Vn), want_lse=True), want)
    big = torch.full((3, B, H, T + 50, D), math.nan, dtype=dtype, device=DEV)
    big[1, :, :, :T] = K
    big2 = torch.full_like(big, math.nan)
    big2[1, :, :, :T] = V
    A.check(lagkv.attend(q, big[1, :, :, :T], big2[1, :, :, :T], Kn, Vn), want)
    odd = torch.full((B, H, T, D + 3), math.nan, dtype=dtype, device=DEV)
    odd2 = odd.clone()
    odd[..., 1:D + 1], odd2[..., 1:D + 1] = K, V
    room = torch.full((B, N + 1, H * G, D + 5), 7.0, dtype=dtype, device=DEV)
    out = room[:, :N, :, 2:D + 2].transpose(1, 2)
    got = lagkv.attend(q, odd[..., 1:D + 1], odd2[..., 1:D + 1], Kn, Vn, out=out)
    A.check(got, want)
    assert got.out is out
    assert bool((room[:, N] == 7).all()) and bool((room[..., :2] == 7).all()) and bool((room[..., D + 2:] == 7).all())
    shared = A.attend(q, K[:1].expand(B, -1, -1, -1), V[:1].expand(B, -1, -1, -1), Kn, Vn)
    A.check(lagkv.attend(q, K[:1].expand(B, H, T, D), V[:1].expand(B, H, T, D), Kn, Vn), shared)
    one = A.attend(q[:, :, :1].expand(-1, -1, N, -1), K, V, Kn, Vn)
    A.check(lagkv.attend(q[:, :, :1].expand(-1, -1, N, -1), K, V, Kn, Vn), one)


def test_offsets_beyond_32_bits():
    """Rows 2^32 bytes and more from the tensor's first: a cache of 2 GiB elements, one row in 4096 of it given."""
    D, T, far = 128, 40, 1 << 26
    big = torch.empty(T * far, dtype=BF, device=DEV)            # 5 GiB
    K = big.as_strided((1, 1, T, D), (0, 0, far, 1))
    V = big.as_strided((1, 1, T, D), (0, 0, far, 1), storage_offset=far // 2)
    k, v = rand(1, 1, T, D, dtype=BF, seed=1), rand(1, 1, T, D, dtype=BF, seed=2)
    K.copy_(k)
    V.copy_(v)
    q = rand(1, 4, 1, D, dtype=BF, seed=3)
    A.check(lagkv.attend(q, K, V, want_lse=True), A.attend(q, k, v))
    lo, hi = lagkv.block_bounds(K, 16)
    wl, wh = A.bounds(k, 16)
    assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
    blocks = torch.tensor([2, 0], dtype=torch.int32, device=DEV).view(1, 1, 1, 2)
    A.check(lagkv.attend_blocks(q, K, V, blocks, 16, want_lse=True), A.attend(q, k, v, blocks=blocks, block=16))
    del big, K, V


def test_a_strong_row_beside_many_weak_ones():
    """A row of logit 17 over 2^17 of logit 0 has 99.5 % of the weight; binary16 alone could not hold the others'."""
    T, D = 1 << 17, 64
    K = torch.zeros(1, 1, T, D, dtype=HF, device=DEV)
    V = torch.ones(1, 1, T, D, dtype=HF, device=DEV)
    q = torch.zeros(1, 1, 1, D, dtype=HF, device=DEV)
    q[..., 0], K[0, 0, 777, 0] = 8.0, 17.0
    V[0, 0, 777] = 0.0
    got = lagkv.attend(q, K, V, scale=0.125, want_lse=True)
    rest = (T - 1) * math.exp(-17.0)
    want = rest / (1 + rest)
    # x is exact; exp and the sums in fp32, the result in 11 bits
    assert float(abs(got.out.double() - want).max()) <= want * (2.0 ** -11 + 2.0 ** -16)
    assert abs(float(got.lse) - (17 + math.log1p(rest))) <= 2.0 ** -18


def test_scale_and_large_logits():
    q, K, V, Kn, Vn = problem(FL, 1, 2, 2, 3, 64, 70, "chain", seed=21)
    for scale in (0.0, -0.3, 4.0):
        A.check(lagkv.attend(q, K, V, Kn, Vn, scale=scale, want_lse=True), A.attend(q, K, V, Kn, Vn, scale=scale), str(scale))
    q, K = q.to(BF), K.to(BF) * 30
    A.check(lagkv.attend(q, K, V.to(BF), want_lse=True), A.attend(q, K, V.to(BF)))


def test_results_do_not_change_from_call_to_call_and_workspace_is_what_is_asked_for():
    q, K, V, Kn, Vn = problem(BF, 1, 2, 4, 3, 128, 5000, "chain", seed=30)
    a = lagkv.attend(q, K, V, Kn, Vn, want_lse=True)
    p = lagkv.AttendParams(1, 2, 4, 3, 128, lagkv.BF16, 0, 0, 5000, 0.1)
    need = lagkv.load().lagkv_attend_workspace_bytes(p)
    assert need > 0
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        b = lagkv.attend(q, K, V, Kn, Vn, want_lse=True, ws=ws[:need])
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    assert bool((ws[need:] == 0x5a).all())
    with pytest.raises(lagkv.LagKVError) as e:
        lagkv.attend(q, K, V, Kn, Vn, ws=ws[:need - 1])
    assert e.value.status == lagkv.EWORKSPACE


BLOCKED = [  # B, H, G, N, D, T, block, k, new
    (1, 1, 1, 1, 64, 1, 16, 1, "none"),
    (2, 2, 4, 1, 128, 517, 16, 7, "chain"),
    (1, 2, 4, 1, 128, 517, 64, 20, "chain"),     # more entries than blocks
    (1, 1, 7, 5, 80, 300, 32, 3, "tree"),
    (2, 1, 20, 3, 96, 400, 128, 2, "chain"),
    (1, 2, 2, 9, 256, 200, 16, 5, "tree"),
    (1, 1, 3, 2, 41, 150, 16, 4, "tree"),
    (1, 1, 4, 2, 128, 4000, 1024, 3, "chain"),
    (1, 1, 4, 1, 128, 9000, 64, 100, "chain"),   # in pieces
    (1, 1, 70, 1, 64, 100, 16, 3, "none"),
]


@pytest.mark.parametrize("dtype", [BF, HF, FL], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", BLOCKED, ids=lambda s: "x".join(map(str, s)))
def test_bounds_select_and_attend_blocks(size, dtype):
    """The three as they are used, each against its plain form on what the one before it gave."""
    B, H, G, N, D, T, block, k, new = size
    print("[gpu-test] blocks", size, dtype, flush=True)
    q, K, V, Kn, Vn = problem(dtype, B, H, G, N, D, T, new, seed=T)
    parents = tree(N, T) if new == "tree" else None
    lengths = torch.tensor([T, T // 2][:B], dtype=torch.int32, device=DEV) if B > 1 else None
    lo, hi = lagkv.block_bounds(K, block, lengths)
    wl, wh = A.bounds(K, block, lengths)
    assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
    first, last = (1, 1) if k > 2 else (0, 0)
    blocks = lagkv.select_blocks(q, lo, hi, T, block, k, first, last, lengths)
    assert torch.equal(blocks.cpu(), A.select(q, lo, hi, T, block, k, first, last, lengths))
    got = lagkv.attend_blocks(q, K, V, blocks, block, Kn, Vn, parents, lengths, want_lse=True)
    A.check(got, A.attend(q, K, V, Kn, Vn, parents, lengths, blocks=blocks.cpu(), block=block), str(size))


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
def test_long_lists_of_many_tokens(dtype):
    """More steps of a list than a wavefront reads entries for at once, in lists that are not cut into pieces."""
    B, H, N, T, block, k = 8, 8, 8, 9000, 64, 140
    q, K, V, Kn, Vn = problem(dtype, B, H, 1, N, 32, T, "chain", seed=44)
    g = torch.Generator().manual_seed(3)
    blocks = torch.rand(B, H, N, 141, generator=g).argsort(-1)[..., :k].to(torch.int32)
    got = lagkv.attend_blocks(q, K, V, blocks.to(DEV), block, Kn, Vn, want_lse=True)
    one = slice(3, 4)
    want = A.attend(q[one], K[one], V[one], Kn[one], Vn[one], blocks=blocks[one], block=block)
    A.check(lagkv.Attended(got.out[one], got.lse[one]), want)


def test_nothing_to_do_and_the_output_in_place_of_the_queries():
    q, K, V, Kn, Vn = problem(BF, 2, 2, 4, 0, 64, 50, "chain", seed=45)
    got = lagkv.attend(q, K, V, Kn, Vn, want_lse=True)
    assert got.out.shape == (2, 8, 0, 64) and got.lse.shape == (2, 8, 0)
    for N, T in ((1, 50), (3, 4000), (40, 500)):
        q, K, V, Kn, Vn = problem(BF, 2, 2, 4, N, 64, T, "chain", seed=46)
        want = A.attend(q, K, V, Kn, Vn)
        assert lagkv.attend(q, K, V, Kn, Vn, out=q).out is q
        A.check(lagkv.Attended(q, None), want)


def test_two_threads():
    """Calls from two threads, each on a stream of its own."""
    import threading
    sets = [problem(BF, 1, 2, 4, 3, 128, 3000, "chain", seed=47 + i) for i in range(2)]
    want = [lagkv.attend(*s).out for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                out = lagkv.attend(*sets[i]).out
            torch.cuda.current_stream().synchronize()
            if not torch.equal(out, want[i]):
                wrong.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


def test_all_blocks_are_all_rows():
    q, K, V, Kn, Vn = problem(BF, 2, 2, 4, 3, 128, 333, "chain", seed=41)
    lo, hi = lagkv.block_bounds(K, 32)
    blocks = lagkv.select_blocks(q, lo, hi, 333, 32, 11)
    A.check(lagkv.attend_blocks(q, K, V, blocks, 32, Kn, Vn, want_lse=True), A.attend(q, K, V, Kn, Vn))


def test_lists_that_name_no_block_or_one_twice():
    T, block = 100, 16
    q, K, V, _, _ = problem(BF, 2, 1, 4, 1, 64, T, "none", seed=50)
    K[1, :, 40:], V[1, :, 40:] = math.nan, math.nan
    lengths = torch.tensor([T, 40], dtype=torch.int32, device=DEV)
    big = (1 << 31) - 1
    lists = [[-1, -1, -1, -1], [6, 7, big, -big], [3, 3, 1, -1], [-1, 2, -1, 0]]
    for row in lists:
        blocks = torch.tensor([row, row], dtype=torch.int32, device=DEV).view(2, 1, 1, 4)
        got = lagkv.attend_blocks(q, K, V, blocks, block, lengths=lengths, want_lse=True)
        A.check(got, A.attend(q, K, V, lengths=lengths, blocks=blocks.cpu(), block=block), str(row))
    # with a token of its own a query that lists nothing sees itself
    Kn, Vn = K[:, :, :1].clone(), V[:, :, :1].clone()
    got = lagkv.attend_blocks(q, K, V, torch.full((2, 1, 1, 4), -1, dtype=torch.int32, device=DEV), block, Kn, Vn, lengths=lengths)
    assert torch.equal(got.out, Vn.expand(2, 4, 1, 64))


def test_bounds_update_leaves_the_blocks_before_it():
    K = rand(2, 2, 210, 40, dtype=HF, seed=60)
    lo, hi = lagkv.block_bounds(K, 16)
    lo0, hi0 = lo.clone(), hi.clone()
    K[:, :, 150:] *= 3
    K[:, :, :100] = 9                                    # not to be seen
    lengths = torch.tensor([210, 155], dtype=torch.int32, device=DEV)
    got = lagkv.block_bounds(K, 16, lengths, start=150, out=(lo, hi))
    assert got[0] is lo and torch.equal(lo[:, :, :9], lo0[:, :, :9]) and torch.equal(hi[:, :, :9], hi0[:, :, :9])
    wl, wh = A.bounds(K, 16, lengths)
    assert torch.equal(lo.cpu()[:, :, 9:], wl[:, :, 9:]) and torch.equal(hi.cpu()[:, :, 9:], wh[:, :, 9:])
    before = lo.clone()
    lagkv.block_bounds(K, 16, start=210, out=(lo, hi))    # nothing behind the last row
    assert torch.equal(lo, before)


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
def test_bounds_between_other_rows(dtype):
    """Bounds in buffers with room, one layer of several, and read from there."""
    T, block = 300, 32
    K, q = rand(2, 3, T, 72, dtype=dtype, seed=61), rand(2, 6, 2, 72, dtype=dtype, seed=62)
    room = torch.full((2, 4, 3, 15, 75), 5.0, dtype=dtype, device=DEV)
    lo, hi = room[0, 1:3, :, 2:12, 1:73], room[1, 1:3, :, 2:12, 1:73]
    lagkv.block_bounds(K, block, out=(lo, hi))
    wl, wh = A.bounds(K, block)
    assert torch.equal(lo.cpu(), wl) and torch.equal(hi.cpu(), wh)
    for n in (1, 2):
        got = lagkv.select_blocks(q[:, :, :n], lo, hi, T, block, 4)
        assert torch.equal(got.cpu(), A.select(q[:, :, :n], wl, wh, T, block, 4))
    q5 = rand(2, 6, 5, 72, dtype=dtype, seed=63)
    assert torch.equal(lagkv.select_blocks(q5, lo, hi, T, block, 4).cpu(), A.select(q5, wl, wh, T, block, 4))
    lo.fill_(5.0), hi.fill_(5.0)
    assert bool((room == 5).all())


def test_equal_scores_go_to_the_lower_block():
    """Blocks of equal bounds, and of scores 0 and -0: the lower index is taken."""
    lo = torch.ones(1, 1, 700, 16, device=DEV)
    hi = lo * 2
    hi[0, 0, 500] = 3.0
    q = rand(1, 2, 3, 16, dtype=FL, seed=70).abs()
    got = lagkv.select_blocks(q, lo, hi, 700 * 16, 16, 5)
    assert torch.equal(got.cpu(), torch.tensor([0, 1, 2, 3, 500], dtype=torch.int32).expand(1, 1, 3, 5))
    q = torch.zeros(1, 2, 1, 16, device=DEV)
    q[0, 1] = -0.0
    lo[0, 0, ::2] = -1.0
    got = lagkv.select_blocks(q, lo, hi, 700 * 16, 16, 300, 0, 2)
    assert got[0, 0, 0].tolist() == list(range(298)) + [698, 699]


@pytest.mark.parametrize("nb,k", [(70, 33), (512, 1), (513, 200), (2049, 64), (8200, 500), (20000, 4096)])
@pytest.mark.parametrize("kind", ["normal", "near", "far", "few", "one", "huge", "wide", "none"])
def test_scores_that_are_hard_to_part(nb, k, kind):
    """Scores that differ in their last bits beside some far away, few distinct ones, the largest range, and some that are no
    numbers ("huge": of infinite bounds; they are q times a bound of either sign, 0 and infinity among them)."""
    g = torch.Generator().manual_seed(nb + k)
    x = torch.randn(nb, generator=g)
    if kind == "near":
        x = 1 + torch.randint(0, 9, (nb,), generator=g) * 2.0 ** -23
    elif kind == "far":
        x = torch.where(torch.rand(nb, generator=g) < 0.9, 1 + torch.randint(0, 99, (nb,), generator=g) * 2.0 ** -23, -3e38 * torch.rand(nb, generator=g))
    elif kind == "few":
        x = torch.randint(-2, 3, (nb,), generator=g).float() * 0.5
    elif kind == "one":
        x = torch.full((nb,), -2.5)
    elif kind == "huge":
        x = x * 3e38 / x.abs().max()
    elif kind == "wide":
        x = x / x.abs().max() * 3e38
    elif kind == "none":
        x[torch.rand(nb, generator=g) < 0.5] = math.nan
    D, N, block = 8, 5, 16
    bound = torch.zeros(1, 1, nb, D)
    bound[0, 0, :, 0] = x
    q = torch.zeros(1, 1, N, D)
    q[0, 0, :, 0] = 1
    first = min(2, k)
    order = sorted(range(nb), key=lambda j: (j >= first, j < first or (-float(x[j]) if math.isfinite(x[j]) else math.inf), j))
    want = torch.tensor(sorted(order[:k]), dtype=torch.int32)
    for n in (1, N):
        got = lagkv.select_blocks(q[:, :, :n].to(DEV), bound.to(DEV), bound.to(DEV), nb * block, block, k, first).cpu()
        assert bool((got == want).all()), (kind, n)


@pytest.mark.parametrize("dtype", [BF, FL], ids=["bf16", "f32"])
def test_selection_at_size(dtype):
    """Thousands of blocks, several tokens, every count of heads of a group; near the border scores are close."""
    for G, N, nb, k in [(1, 1, 5000, 64), (4, 3, 1030, 1), (6, 2, 2049, 700), (3, 17, 130, 129)]:
        K = rand(1, 2, nb * 16 - 5, 64, dtype=dtype, seed=nb)
        lo, hi = lagkv.block_bounds(K, 16)
        q = rand(1, 2 * G, N, 64, dtype=dtype, seed=nb + 1)
        got = lagkv.select_blocks(q, lo, hi, nb * 16 - 5, 16, k)
        assert torch.equal(got.cpu(), A.select(q, lo, hi, nb * 16 - 5, 16, k)), (G, N, nb, k)


def test_other_streams_and_two_calls_at_once():
    q, K, V, Kn, Vn = problem(BF, 1, 2, 4, 3, 128, 5000, "chain", seed=80)
    q2, K2, V2, Kn2, Vn2 = problem(BF, 1, 2, 4, 3, 128, 5000, "chain", seed=81)
    want, want2 = lagkv.attend(q, K, V, Kn, Vn).out, lagkv.attend(q2, K2, V2, Kn2, Vn2).out
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s1):
            a = lagkv.attend(q, K, V, Kn, Vn).out
        with torch.cuda.stream(s2):
            b = lagkv.attend(q2, K2, V2, Kn2, Vn2).out
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want2)


def test_captured_steps_replayed():
    """A decode step in a graph (bounds of the last rows, selection, attention over blocks and over all rows): lengths live on the
    device, so that one graph serves a growing cache.  Two graphs, with eager work and synchronisation between replays."""
    B, H, G, D, cap, block, k = 2, 2, 4, 128, 4096, 32, 8
    K, V = rand(B, H, cap, D, dtype=BF, seed=90), rand(B, H, cap, D, dtype=BF, seed=91)
    lo, hi = lagkv.block_bounds(K, block)
    lengths = torch.tensor([100, 50], dtype=torch.int32, device=DEV)
    graphs = []
    for i in range(2):
        q, Kn, Vn = rand(B, H * G, 1, D, dtype=BF, seed=92 + i), rand(B, H, 1, D, dtype=BF, seed=94 + i), rand(B, H, 1, D, dtype=BF, seed=96 + i)

        def step(q=q, Kn=Kn, Vn=Vn):
            lagkv.block_bounds(K, block, lengths, start=0, out=(lo, hi))
            blocks = lagkv.select_blocks(q, lo, hi, cap, block, k, 1, 1, lengths)
            some = lagkv.attend_blocks(q, K, V, blocks, block, Kn, Vn, lengths=lengths, want_lse=True)
            every = lagkv.attend(q, K, V, Kn, Vn, lengths=lengths, want_lse=True)
            return blocks, some.out, some.lse, every.out, every.lse

        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step()
        graphs.append((g, got, step))
    for lens in ([100, 50], [101, 0], [4096, 1], [3000, 2999]):
        lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        want = [step() for _, _, step in graphs]
        torch.cuda.synchronize()
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, got, _), w in zip(graphs, want):
            for x, y in zip(got, w):
                assert torch.equal(x, y), lens
