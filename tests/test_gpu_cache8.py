"""The 8-bit cache object on tensors of every one-byte type, and its refusals."""
import pytest
import torch

from _cases8 import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("payload", [torch.uint8, torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("scales", [torch.uint8, torch.int8, torch.float8_e8m0fnu])
def test_values_go_by_the_bytes(payload, scales):
    from paper_2609_02897_gb300 import asd8
    case = Case(1, [4], [100], Hkv=2, D=64, garbage=False).fill()
    plain = case.cache()
    other = asd8.Cache8(case.dims(), k=plain.k.view(payload), v=plain.v.view(payload),
                        k_exp=plain.k_exp.view(scales), v_exp=plain.v_exp.view(scales))
    for which, want in zip("kv", case.values()):
        got = other.values(which)
        assert torch.equal(got, plain.values(which))
        assert (got.double().cpu().numpy()[:, :, :100] == want[:, :, :100]).all()


def test_refusals():
    from paper_2609_02897_gb300 import asd8
    case = Case(1, [4], [100], Hkv=2, D=64).fill()
    c = case.cache()
    for kw in (dict(k=c.k.to(torch.int16)), dict(k=c.k[:, :, :-1]), dict(v_exp=c.v_exp[..., :-1]),
               dict(v=c.v.cpu()), dict(k=c.k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            asd8.Cache8(case.dims(), **kw)
