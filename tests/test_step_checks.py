"""A step's tensors are checked once per set: what lies at a remembered address later is another tensor. No device needed."""
import pytest
import torch

from paper_2601_12784_amd import binding as B


class OnGpu(torch.Tensor):
    is_cuda = True


def tensors(b=3, hq=4, hkv=2, d=64, n=5, fp8=False):
    shapes = dict(q=((b, hq, d), torch.bfloat16), block_table=((b, 4), torch.int32), out=((b, hq, d), torch.float32),
                  lse=((b, hq), torch.float32))
    if fp8:
        shapes.update({x: ((n, hkv, 16 * d), torch.uint8) for x in ("k_pool", "v_pool")},
                      **{x: ((n, hkv), torch.float32) for x in ("k_scale", "v_scale")})
    else:
        shapes.update(k_pool=((n, hkv, d // 8, 16, 8), torch.bfloat16), v_pool=((n, hkv, d, 16), torch.bfloat16))
    return {name: torch.zeros(shape, dtype=dtype).as_subclass(OnGpu) for name, (shape, dtype) in shapes.items()}


def other_type(t):
    return t.view({torch.bfloat16: torch.float16, torch.float32: torch.int32, torch.int32: torch.float32,
                   torch.uint8: torch.int8}[t.dtype])


def shorter(t):
    return t[:-1]


def strided(t):
    return torch.as_strided(t, t.shape, (0, *t.stride()[1:]))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("change", [other_type, shorter, strided])
@pytest.mark.parametrize("remembered", [256, 4, 0])
def test_another_tensor_at_a_remembered_address_is_checked(fp8, change, remembered):
    attn = B.DecodeAttention.__new__(B.DecodeAttention)
    attn.hq, attn.hkv, attn.d, attn._checked, attn._checks_left = 4, 2, 64, {}, remembered

    def check(x):
        attn._check_tensors(x["q"], x["k_pool"], x["v_pool"], x["block_table"], x["out"], x["lse"],
                            (x["k_scale"], x["v_scale"]) if fp8 else None)

    good = tensors(fp8=fp8)
    check(good)
    check(good)
    for name in good:
        if change is shorter and name in ("q", "k_pool"):
            continue      # they say what the others' shapes have to be
        bad = dict(good, **{name: change(good[name])})
        assert bad[name].data_ptr() == good[name].data_ptr()
        with pytest.raises(ValueError):
            check(bad)
    check(good)
