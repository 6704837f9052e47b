"""QuantizedCache refuses what its operators would refuse when the first rows become final: before any row is in it."""
import pytest
import torch

from paper_2504_04704_amd import lagkv


def cache(D=64, block=64, code=torch.int8, capacity=256, dtype=torch.bfloat16):
    return lagkv.QuantizedCache(1, 2, D, capacity, 4, 32, 0.5, block, code, dtype=dtype, device="cpu")


@pytest.mark.parametrize("kw,status", [(dict(block=0), lagkv.EINVAL), (dict(block=8), lagkv.EINVAL), (dict(block=100), lagkv.EINVAL), (dict(block=2048), lagkv.EINVAL),
                                       (dict(block=-16), lagkv.EINVAL), (dict(D=8), lagkv.ESHAPE), (dict(D=264), lagkv.ESHAPE)], ids=str)
def test_limits(kw, status):
    with pytest.raises(lagkv.LagKVError) as e:
        cache(**kw)
    assert e.value.status == status


def test_codes():
    with pytest.raises(TypeError):
        cache(code=torch.uint8)


def test_what_is_taken():
    for kw in (dict(), dict(block=16, D=16), dict(block=1024, D=256, code=torch.float8_e4m3fn), dict(capacity=0)):
        x = cache(**kw)
        assert x.length == 0 and x.rows.block == kw.get("block", 64)
