"""Tensors that carry a tangent are refused, as those that ask for a gradient are: it would be lost."""
import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2504_04704_amd import lagkv


def test_tangents_are_seen():
    x = torch.zeros(2, 3)
    lagkv._no_grad(x, None)
    with fw.dual_level():
        lagkv._no_grad(x, None)
        dual = fw.make_dual(x, torch.ones_like(x))
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(RuntimeError, match="forward-mode"):
                lagkv._no_grad(None, dual)
        lagkv._no_grad(fw.unpack_dual(dual).primal)
    lagkv._no_grad(dual)                                       # (its level is gone, and the tangent with it)


@pytest.mark.gpu
def test_dual_tensors_are_refused():
    g = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to("cuda:0")
    q, K, Kn = g(1, 4, 2, 64), g(1, 2, 50, 64), g(1, 2, 2, 64)
    blocks = torch.zeros(1, 2, 2, 1, dtype=torch.int32, device="cuda:0")
    lo, hi = lagkv.block_bounds(K, 16)
    want = lagkv.attend(q, K, K, Kn, Kn).out
    calls = [(lagkv.attend, (q, K, K, Kn, Kn), {}, range(5)), (lagkv.attend_blocks, (q, K, K, blocks, 16, Kn, Kn), {}, (0, 1, 2, 5, 6)),
             (lagkv.block_bounds, (K, 16), {}, (0,)), (lagkv.select_blocks, (q, lo, hi, 50, 16, 2), {}, (0, 1, 2))]
    with fw.dual_level():
        for f, args, kw, which in calls:
            for i in which:
                a = list(args)
                a[i] = fw.make_dual(a[i], torch.ones_like(a[i]))
                if f is lagkv.attend and i in (1, 2, 3, 4):    # (K and V, and K_new and V_new, share their layout)
                    assert a[i].stride() == args[i].stride()
                with pytest.raises(RuntimeError, match="forward-mode"):
                    f(*a, **kw)
                with torch.no_grad(), pytest.raises(RuntimeError, match="forward-mode"):
                    f(*a, **kw)
        assert torch.equal(lagkv.attend(q, K, K, Kn, Kn).out, want)
