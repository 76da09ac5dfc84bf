"""Rotary's frequencies, table and refusals, without a GPU."""
import math

import pytest
import torch

from paper_2511_01282_gb300 import rotary


def test_frequencies():
    f = rotary.frequencies(8, 10000.0)
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(rotary.frequencies(8, factor=4.0), f / 4)
    # waves of 2 pi / f positions: into 100 they fit 15.9, 1.59, 0.159 times
    s = rotary.frequencies(8, factor=4.0, trained=100, low=1.0, high=4.0)
    fit = 100 * 0.1 / (2 * math.pi)
    keep = (fit - 1) / 3
    want = [1.0, 0.1 * (keep + (1 - keep) / 4), 0.01 / 4, 0.001 / 4]
    assert torch.allclose(s, torch.tensor(want, dtype=torch.float64), rtol=1e-14)
    for bad in (dict(rot=0), dict(rot=7), dict(rot=8, base=0.0), dict(rot=8, factor=-1.0), dict(rot=8, low=4.0, high=4.0)):
        with pytest.raises(ValueError):
            rotary.frequencies(**bad)


def test_turns():
    f = torch.tensor([0.0, math.pi, -math.pi / 2, 1.0, 7.0], dtype=torch.float64)
    w = [x % 2 ** 64 for x in rotary.turns(f).tolist()]
    assert w[0] == 0 and abs(w[1] - 2 ** 63) < 2 ** 12 and abs(w[2] - 3 * 2 ** 62) < 2 ** 12
    # 1 / (2 pi) = 0.15915494309189533576888376337251436... and 7 / (2 pi) less a turn
    assert abs(w[3] - 2935890503282001226) <= 1 and abs(w[4] - (7 * 2935890503282001226 - 2 ** 64)) <= 7
    with pytest.raises(ValueError):
        rotary.turns(torch.tensor([math.inf]))


def test_refusals():
    for bad in (dict(D=60), dict(D=520), dict(D=64, rot=66), dict(D=64, rot=7), dict(D=64, layout="pairs"),
                dict(D=64, freq=torch.ones(31, dtype=torch.float64))):
        with pytest.raises(ValueError):
            rotary.Rotary(**dict(dict(device="cpu"), **bad))
    r = rotary.Rotary(64, device="cpu")
    x, pos = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for q, k, p, out, word in [(None, None, pos, None, "q or k"), (x.float(), None, pos, None, "bfloat16"), (x, x[:2], pos, None, "k:"),
                               (x, x.half(), pos, None, "k:"), (x, None, pos[:2], None, "pos"), (x, None, pos.long(), None, "pos"),
                               (x[..., :32], None, pos, None, "q:"), (x, None, pos, (x[:, :1], None), "q:")]:
        with pytest.raises(ValueError, match=word):
            r(q, k, p, out)


def test_results_with_a_gradient_are_new_tensors():
    r = rotary.Rotary(64, device="cpu")
    x, pos = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    leaf = x.clone().requires_grad_()
    for q, k, out in ((leaf, None, (x, None)), (x, leaf, (None, x)), (leaf, x, (leaf, x)), (x, x, (leaf, None))):
        with pytest.raises(ValueError, match="out"):
            r(q, k, pos, out)


def test_frequencies_whose_turns_the_digits_of_pi_do_not_give_are_refused():
    # 2^95 / (2 pi) x 2^64 takes 157 of the table's 166 bits of pi; 10^40 rather more than it has
    for f in (1e40, -1e40, 2.0 ** 96):
        with pytest.raises(ValueError, match="2\\^96"):
            rotary.turns(torch.tensor([1.0, f], dtype=torch.float64))
    two_pi = 2 * rotary.Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
    for f in (2.0 ** 95, -2.0 ** 95 * 1.75):
        want = round(rotary.Fraction(f) / two_pi * 2 ** 64) % 2 ** 64
        assert rotary.turns(torch.tensor([f], dtype=torch.float64)).item() % 2 ** 64 == want
