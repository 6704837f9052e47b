"""quantize() into codes of another kind than those that are asked for is refused, and codes are those of `out` where none are asked for."""
import pytest
import torch

from paper_2504_04704_amd import lagkv

I8, E4 = torch.int8, torch.float8_e4m3fn


@pytest.mark.parametrize("asked,has", [(I8, E4), (E4, I8), (torch.uint8, I8)])
def test_other_codes_are_refused(asked, has):
    x = torch.zeros(1, 2, 40, 64)
    with pytest.raises(ValueError, match="codes"):
        lagkv.quantize(x, x, 16, asked, out=lagkv.Quantized.empty(1, 2, 40, 64, 16, has, "cpu"))


@pytest.mark.gpu
@pytest.mark.parametrize("use_native", [True, False])
@pytest.mark.parametrize("has", [I8, E4], ids=["int8", "e4m3"])
def test_on_the_device(has, use_native):
    K = torch.randn(1, 2, 40, 64, generator=torch.Generator().manual_seed(1)).to("cuda:0")
    lagkv.load()
    native = lagkv._native
    assert native is not None
    lagkv._native = native if use_native else None
    try:
        out = [lagkv.Quantized.empty(1, 2, 40, 64, 16, has, "cuda:0") for _ in range(3)]
        for x in out:
            x.K.view(I8).fill_(99)
        with pytest.raises(ValueError, match="codes"):
            lagkv.quantize(K, K, 16, E4 if has == I8 else I8, out=out[0])
        assert bool((out[0].K.view(I8) == 99).all())
        lagkv.quantize(K, K, 16, out=out[1])
        lagkv.quantize(K, K, 16, has, out=out[2])
        want = lagkv.quantize(K, K, 16, has)
        for x in out[1:]:
            assert torch.equal(x.K.view(I8), want.K.view(I8)) and torch.equal(x.V_scale, want.V_scale)
        assert lagkv.quantize(K, K, 16).K.dtype == I8
    finally:
        lagkv._native = native
