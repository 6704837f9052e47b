"""Refusals of the operators that read a cache, all of them before any device work, and the layout of their parameters."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

from paper_2504_04704_amd import lagkv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000            # an address that is never read: every call below is refused first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lagkv.lib_path()):
        from paper_2504_04704_amd import build
        build.build_library(verbose=False)
    return lagkv.load()


def params(**kw):
    d = dict(B=2, H=2, G=4, N=3, D=64, dtype=lagkv.BF16, block=32, n_blocks=0, T=1000, scale=0.125)
    d.update({k: v for k, v in kw.items() if k in d})
    p = lagkv.AttendParams(**d)
    B, H, G, N, D, T = (d[x] for x in ("B", "H", "G", "N", "D", "T"))
    p.q_stride[:] = kw.get("q", (H * G * N * D, N * D, D))
    p.out_stride[:] = kw.get("out", (H * G * N * D, N * D, D))
    p.kv_stride[:] = kw.get("kv", (H * T * D, T * D, D))
    p.new_stride[:] = kw.get("new", (H * N * D, N * D, D))
    p.parents_stride_b = kw.get("psb", 0)
    return p


def attend(lib, p, Q=P, K=P, V=P, lengths=None, Kn=P, Vn=P, parents=None, out=P, lse=None, ws=P, n=1 << 40):
    return lib.lagkv_attend(C.byref(p) if p is not None else None, Q, K, V, lengths, Kn, Vn, parents, out, lse, ws, n, None)


def attend_blocks(lib, p, blocks=P, **kw):
    a = dict(Q=P, K=P, V=P, lengths=None, Kn=None, Vn=None, parents=None, out=P, lse=None, ws=P, n=1 << 40)
    a.update(kw)
    return lib.lagkv_attend_blocks(C.byref(p), a["Q"], a["K"], a["V"], a["lengths"], blocks, a["Kn"], a["Vn"], a["parents"],
                                   a["out"], a["lse"], a["ws"], a["n"], None)


def test_layout(tmp_path):
    src = tmp_path / "l.c"
    names = ["H", "dtype", "block", "n_blocks", "T", "scale", "q_stride_b", "kv_stride_b", "new_stride_b", "out_stride_n", "parents_stride_b"]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "lagkv.h"\nint main(void){printf("%zu", sizeof(lagkv_attend_params));' +
                   "".join(f'printf(" %zu", offsetof(lagkv_attend_params, {n}));' for n in names) + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()]
    A = lagkv.AttendParams
    assert got == [C.sizeof(A), A.H.offset, A.dtype.offset, A.block.offset, A.n_blocks.offset, A.T.offset, A.scale.offset,
                   A.q_stride.offset, A.kv_stride.offset, A.new_stride.offset, A.out_stride.offset + 16, A.parents_stride_b.offset]


def test_attend_refuses(lib):
    E, S, D = lagkv.EINVAL, lagkv.ESHAPE, lagkv.EDTYPE
    assert attend(lib, None) == E
    assert attend(lib, params(N=0), Q=None, out=None) == lagkv.OK           # nothing to do
    for kw, want in [(dict(dtype=3), D), (dict(dtype=-1), D), (dict(B=0), S), (dict(H=0), S), (dict(G=0), S), (dict(N=-1), S),
                     (dict(D=7), S), (dict(D=257), S), (dict(T=-1), S), (dict(T=(1 << 31) - 1), S), (dict(scale=math.inf), E),
                     (dict(scale=math.nan), E), (dict(scale=1e39), E), (dict(B=1 << 20, H=1 << 10), S), (dict(G=1 << 16, N=1 << 16), S),
                     (dict(q=(-1, 0, 0)), S), (dict(kv=(0, -1, 0)), S), (dict(new=(0, 0, -1)), S), (dict(psb=-1), S),
                     # rows of the output on one another
                     (dict(out=(0, 192, 64)), S), (dict(out=(1536, 192, 63)), S), (dict(out=(1536, 0, 64)), S),
                     (dict(out=(1536, 191, 64)), S), (dict(out=(-1536, 192, 64)), S)]:
        assert attend(lib, params(**kw)) == want, kw
    ok = params()
    for kw in [dict(Q=None), dict(K=None), dict(V=None), dict(out=None), dict(Kn=None), dict(Vn=None), dict(Q=P + 1), dict(K=P + 1),
               dict(Vn=P + 1), dict(out=P + 1), dict(lse=P + 2), dict(lengths=P + 2), dict(parents=P + 2),
               dict(parents=P, Kn=None, Vn=None)]:
        assert attend(lib, ok, **kw) == E, kw
    assert attend(lib, params(N=257), parents=P) == S                       # a tree of more tokens than it takes
    need = lib.lagkv_attend_workspace_bytes(C.byref(params(T=100000)))
    assert need > 0 and need % 256 == 0
    for kw in [dict(ws=None), dict(n=need - 1), dict(ws=P + 8)]:
        assert attend(lib, params(T=100000), **kw) == lagkv.EWORKSPACE, kw
    assert lib.lagkv_attend_workspace_bytes(None) == 0 and lib.lagkv_attend_workspace_bytes(C.byref(params(D=300))) == 0
    # more workgroups than a grid has
    assert attend(lib, params(B=1 << 14, H=1 << 10, G=64, N=1 << 14)) == S


def test_attend_blocks_refuses(lib):
    E = lagkv.EINVAL
    for kw in [dict(block=0), dict(block=8), dict(block=24), dict(block=2048), dict(block=-16), dict(n_blocks=0), dict(n_blocks=-1),
               dict(block=1024, n_blocks=1 << 22)]:
        assert attend_blocks(lib, params(**{"n_blocks": 4, **kw})) == E, kw
    assert attend_blocks(lib, params(n_blocks=4), blocks=None) == E
    assert attend_blocks(lib, params(n_blocks=4), blocks=P + 2) == E
    assert attend_blocks(lib, params(n_blocks=4), Kn=P) == E


def test_bounds_and_selection_refuse(lib):
    E, S = lagkv.EINVAL, lagkv.ESHAPE

    def bounds(p, K=P, lengths=None, start=0, lo=P, hi=P):
        return lib.lagkv_block_bounds(C.byref(p), K, lengths, start, lo, hi, None)

    assert bounds(params(T=0), K=None) == lagkv.OK and bounds(params(), start=1000) == lagkv.OK
    for kw in [dict(K=None), dict(lo=None), dict(hi=None), dict(start=-1), dict(K=P + 1), dict(lengths=P + 1), dict(hi=P + 1)]:
        assert bounds(params(), **kw) == E, kw
    wide = (1 << 20, 1 << 19, 64)
    assert bounds(params()) == S and bounds(params(out=(1 << 20, 1 << 19, 63))) == S and bounds(params(out=(-1, 0, 0))) == S
    assert bounds(params(out=wide, block=12)) == E and bounds(params(kv=(0, 0, -1))) == S and bounds(params(dtype=9)) == lagkv.EDTYPE

    def select(p, Q=P, lo=P, hi=P, lengths=None, first=0, last=0, blocks=P, ws=P, n=1 << 40):
        return lib.lagkv_select_blocks(C.byref(p), Q, lo, hi, lengths, first, last, blocks, ws, n, None)

    ok = params(n_blocks=4)
    assert select(params(n_blocks=4, N=0)) == lagkv.OK
    for kw in [dict(Q=None), dict(lo=None), dict(hi=None), dict(blocks=None), dict(first=-1), dict(last=-1), dict(first=3, last=2),
               dict(first=(1 << 31) - 1, last=(1 << 31) - 1), dict(Q=P + 1), dict(blocks=P + 1)]:
        assert select(ok, **kw) == E, kw
    assert select(params(n_blocks=4, kv=(0, 0, -1))) == S
    assert select(params(n_blocks=0)) == E and select(params(n_blocks=4, block=20)) == E
    need = 8 * 2 * 2 * 3 * 32
    for kw in [dict(ws=None), dict(n=need - 1), dict(ws=P + 8)]:
        assert select(ok, **kw) == lagkv.EWORKSPACE, kw


def test_binding_refuses(lib):
    x = torch.zeros(1, 2, 8, 64)
    with pytest.raises(RuntimeError, match="no CPU path"):
        lagkv.attend(x, x, x)
    with pytest.raises(RuntimeError, match="no CPU path"):
        lagkv.block_bounds(x, 16)
    with pytest.raises(RuntimeError, match="no CPU path"):
        lagkv.select_blocks(x, x, x, 128, 16, 2)
    with pytest.raises(TypeError):
        lagkv.attend(x.double(), x.double(), x.double())
    with pytest.raises(ValueError):
        lagkv.attend(x[0], x, x)
    with pytest.raises(ValueError):
        lagkv.attend(x.transpose(2, 3), x, x)
    with pytest.raises(ValueError):
        lagkv.attend_blocks(x, x, x, None, 16)


@pytest.mark.gpu
def test_binding_refuses_on_device(lib):
    g = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda:0")
    q, K, Kn = g(2, 8, 3, 64), g(2, 2, 50, 64), g(2, 2, 3, 64)
    i32 = lambda *s: g(*s, dtype=torch.int32)
    bad = [dict(q=g(2, 7, 3, 64)), dict(q=g(1, 8, 3, 64)), dict(q=g(2, 8, 3, 32)), dict(q=q.half()), dict(V=g(2, 2, 49, 64)),
           dict(V=K.float()), dict(V_new=None), dict(K_new=g(2, 2, 4, 64), V_new=g(2, 2, 4, 64)), dict(K_new=None, V_new=None, parents=i32(3)),
           dict(parents=i32(4)), dict(parents=i32(3, 3)), dict(parents=g(3, dtype=torch.int64)), dict(lengths=i32(3)),
           dict(lengths=g(2, dtype=torch.int64)), dict(lengths=torch.zeros(2, dtype=torch.int32)), dict(out=g(2, 8, 3, 32)),
           dict(out=q.half()), dict(ws=g(4, dtype=torch.int32))]
    for kw in bad:
        a = dict(q=q, K=K, V=K, K_new=Kn, V_new=Kn)
        a.update(kw)
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            lagkv.attend(**a)
    for kw in [dict(blocks=i32(2, 2, 3)), dict(blocks=i32(2, 2, 2, 4)), dict(blocks=i32(2, 2, 3, 0)), dict(block=17)]:
        a = dict(q=q, K=K, V=K, blocks=i32(2, 2, 3, 4), block=16)
        a.update(kw)
        with pytest.raises((ValueError, lagkv.LagKVError)):
            lagkv.attend_blocks(**a)
    with pytest.raises(lagkv.LagKVError):
        lagkv.attend(q, K, K, out=g(1, 8, 3, 64).expand(2, 8, 3, 64))
    with pytest.raises(ValueError):
        lagkv.block_bounds(K, 16, start=5)
    with pytest.raises(ValueError):
        lagkv.block_bounds(K, 16, out=(g(2, 2, 3, 64), g(2, 2, 4, 64)))
    with pytest.raises(ValueError):
        lagkv.select_blocks(q, g(2, 2, 3, 64), g(2, 2, 3, 64), 50, 16, 2)
    with pytest.raises(lagkv.LagKVError):
        lagkv.select_blocks(q, g(2, 2, 4, 64), g(2, 2, 4, 64), 50, 16, 2, first=2, last=1)
    w = q.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="no backward"):
        lagkv.attend(w, K, K)
    with torch.no_grad():
        lagkv.attend(w, K, K)
