"""The operators of a cache in 8 bits on streams of their own, under graph capture, on large offsets, through both bindings."""
import threading

import pytest
import torch

import attend_util as A
import quant_util as Q
from paper_2504_04704_amd import lagkv
from test_attend_quantized import BF, CODES, DEV, E4, FL, HF, I8, problem, rand, stored, tree

pytestmark = pytest.mark.gpu


def all_of(x):
    return [t.view(I8) if t.dtype == E4 else t for t in (x.K, x.V, x.K_scale, x.V_scale)]


@CODES
def test_a_captured_step(code):
    """Rows written, quantised, attended to and read back in one graph, replayed on other rows with eager work in between."""
    B, H, G, N, D, T, block = 2, 2, 4, 3, 128, 320, 32
    K, V = (torch.empty(B, H, T, D, dtype=BF, device=DEV) for _ in range(2))
    q, Kn, Vn = (torch.empty(B, h, N, D, dtype=BF, device=DEV) for h in (H * G, H, H))
    x, y = (lagkv.Quantized.empty(B, H, 256, D, block, code, DEV) for _ in range(2))

    def fill(seed):
        for i, t in enumerate((K, V, q, Kn, Vn)):
            t.copy_(rand(*t.shape, dtype=BF, seed=seed + i))

    def step(x):
        lagkv.quantize(K[:, :, :256], V[:, :, :256], block, out=x)
        a = lagkv.attend_quantized(q, x, K[:, :, 256:], V[:, :, 256:], Kn, Vn, want_lse=True)
        return a, lagkv.dequantize(x, BF)

    fill(0)
    step(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, back = step(x)
    for seed in (10, 20, 30, 40):
        fill(seed)
        graph.replay()
        want, rows = step(y)
        torch.cuda.synchronize()
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
        assert all(torch.equal(a, b) for a, b in zip(all_of(x), all_of(y))) and torch.equal(back[0], rows[0]) and torch.equal(back[1], rows[1])
        lagkv.attend(q, K, V, Kn, Vn)


def test_two_streams_and_two_threads():
    """Calls side by side, each with a workspace of its own."""
    problems = [problem(BF, c, 2, 2, 4, n, 128, 3000, 50, "chain", 64, seed=s) for c, n, s in ((I8, 1, 1), (E4, 40, 2), (I8, 8, 3), (E4, 1, 4))]
    want = [lagkv.attend_quantized(*p, want_lse=True) for p in problems]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(30):
                    got = lagkv.attend_quantized(*problems[i], want_lse=True)
            stream.synchronize()
            assert torch.equal(got.out, want[i].out) and torch.equal(got.lse, want[i].lse)
        except BaseException as e:
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_the_same_twice():
    """No result depends on the order in which workgroups end."""
    for dtype in (BF, HF, FL):
        p = problem(dtype, I8, 1, 4, 4, 3, 128, 9000, 300, "chain", 64, seed=7)
        first = lagkv.attend_quantized(*p, want_lse=True)
        for _ in range(5):
            again = lagkv.attend_quantized(*p, want_lse=True)
            assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)


@CODES
def test_offsets_beyond_32_bits(code):
    """Codes of more than 4 GiB behind the first row, scales and rows far apart: the last head of a store with long strides."""
    H, D, T, far = 2, 64, 100, (1 << 32) + 4096
    store = torch.empty(far + (T + 8) * D, dtype=I8, device=DEV)
    view = lambda: torch.as_strided(store.view(code), (1, H, T, D), (0, far, D, 1))  # noqa: E731
    other = stored(1, H, T, D, 32, code, 3)
    x = lagkv.Quantized(view(), view(), other.K_scale, other.V_scale, 32)
    store[:T * D].copy_(other.K[0, 0].view(I8).flatten())
    store[far:far + T * D].copy_(other.K[0, 1].view(I8).flatten())
    near = lagkv.Quantized(other.K, other.K, other.K_scale, other.V_scale, 32)
    for N in (1, 40):
        q = rand(1, 4, N, D, dtype=BF, seed=4)
        a, b = lagkv.attend_quantized(q, x, want_lse=True), lagkv.attend_quantized(q, near, want_lse=True)
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    assert torch.equal(lagkv.dequantize(x)[0], lagkv.dequantize(near)[0])
    K = rand(1, H, T, D, dtype=BF, seed=5)
    room = torch.empty(2, far + (T + 8) * D, dtype=I8, device=DEV)
    y = lagkv.Quantized(*(torch.as_strided(r.view(code), (1, H, T, D), (far + T * D, far, D, 1)) for r in room),
                        other.K_scale.clone(), other.V_scale.clone(), 32)
    lagkv.quantize(K, K, 32, out=y)
    want = lagkv.quantize(K, K, 32, code)
    assert torch.equal(y.K.view(I8), want.K.view(I8)) and torch.equal(y.V_scale, want.V_scale)


def test_both_bindings():
    """The native step and ctypes say the same."""
    p = problem(BF, E4, 2, 2, 4, 9, 96, 500, 40, "tree", 32, seed=8)
    parents = tree(9, 3, 2)
    K, V = rand(2, 2, 100, 96, dtype=BF, seed=1), rand(2, 2, 100, 96, dtype=BF, seed=2)
    native, got = lagkv._native, []
    assert native is not None
    for use in (native, None):
        lagkv._native = use
        try:
            a = lagkv.attend_quantized(*p, parents, want_lse=True)
            x = lagkv.quantize(K, V, 32, E4, out=lagkv.Quantized.empty(2, 2, 100, 96, 32, E4, DEV))
            got.append([a.out, a.lse, *all_of(x), *lagkv.dequantize(x, out=(torch.zeros_like(K), torch.zeros_like(V)), start=7)])
        finally:
            lagkv._native = native
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_workspace_that_is_given():
    q, x, *rows = problem(BF, I8, 1, 2, 4, 2, 64, 400, 20, "chain", 32, seed=9)
    want = lagkv.attend_quantized(q, x, *rows)
    p = lagkv.QuantParams(B=1, H=2, G=4, N=2, D=64, dtype=lagkv.BF16, code=lagkv.CODE_INT8, block=32, T=400, R=20, scale=1.0)
    need = lagkv.load().lagkv_attend_quantized_workspace_bytes(p)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    got = lagkv.attend_quantized(q, x, *rows, ws=ws[:need])
    assert torch.equal(got.out, want.out) and bool((ws[need:] == 255).all())
    with pytest.raises(lagkv.LagKVError):
        lagkv.attend_quantized(q, x, *rows, ws=ws[:need - 1])
