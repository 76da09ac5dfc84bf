"""The e4m3 restatement against the type's own conversions, without a GPU."""
import math

import torch

import coded_ref as cr


def test_codes_and_values():
    codes = torch.arange(256, dtype=torch.uint8)
    own = codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(cr.decode(codes).nan_to_num(-1e9), own.nan_to_num(-1e9))
    x = torch.cat([torch.randn(20000, generator=torch.Generator().manual_seed(1)) * s for s in (1e-3, 0.02, 1.0, 60.0)]).clamp(-448, 448)
    mid = (cr.VALUES[1:] + cr.VALUES[:-1]) / 2  # ties
    x = torch.cat([x, mid.float(), -mid.float(), torch.tensor([0.0, -0.0, 448.0, -448.0, math.nan])])
    assert torch.equal(cr.encode(x), x.to(torch.float8_e4m3fn).view(torch.uint8))


def test_exponents():
    for dt, (lo, hi) in cr.RANGE.items():
        assert cr.exponent([0.0], dt) == lo and cr.exponent([math.nan, -math.inf], dt) == lo
        assert cr.exponent([448.0, -1.0], dt) == 0 and cr.exponent([-448.5], dt) == 1 and cr.exponent([224.0], dt) == -1
        assert cr.exponent([torch.finfo(dt).max], dt) == hi
    assert cr.decode(cr.block_codes(torch.tensor([65504.0, -65504.0, 61000.0]).half(), 8, torch.float16)).tolist() == [240.0, -240.0, 240.0]
    most = torch.finfo(torch.bfloat16).max
    assert cr.decode(cr.block_codes(torch.tensor([most, -most]).bfloat16(), 120, torch.bfloat16)).tolist() == [240.0, -240.0]
