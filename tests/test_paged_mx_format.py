"""The definition of the 4-bit format against examples worked out by hand."""
import torch

from paged_mx_reference import quantise, values


def row(*first, fill=0.0):
    x = torch.full((128,), fill, dtype=torch.bfloat16)
    x[:len(first)] = torch.tensor(first, dtype=torch.bfloat16)
    return x


def test_scale_of_a_group():
    for top, byte in ((6.0, 127), (4.0, 127), (3.5, 127), (3.0, 126), (3.484375, 126), (7.0, 128), (6.96875, 127), (8.0, 128), (1.0, 125),
                      (0.0, 2), (2.0 ** -126, 2), (2.0 ** 127 * 1.75, 252), (2.0 ** 127, 252)):
        assert int(quantise(row(top, -top / 4))[1][0]) == byte, top
    codes, scale = quantise(row(1.0, float("nan")))
    assert scale.tolist() == [255, 2, 2, 2] and not codes.any()
    assert quantise(row(float("-inf")))[1].tolist() == [255, 2, 2, 2]


def test_values_go_to_the_nearest_level_and_ties_to_even():
    x = row(6.0, 0.25, 0.26, 0.75, 1.25, 1.26, 1.75, 2.5, 2.52, 3.5, 5.0, 5.03, -0.25, -0.75, 6.9, -6.9)
    codes, scale = quantise(x)
    got = values(codes, scale)[:16].tolist()
    assert int(scale[0]) == 127
    assert got == [6, 0, 0.5, 1, 1, 1.5, 2, 2, 3, 4, 4, 6, 0, -1, 6, -6]
    assert int(codes[6] & 15) == 8      # -0.25: minus zero


def test_rounding_is_within_its_bound():
    g = torch.Generator().manual_seed(5)
    x = (torch.randn(4000, 128, generator=g) * torch.exp(3 * torch.randn(4000, 1, generator=g))).to(torch.bfloat16)
    codes, scale = quantise(x)
    back = values(codes, scale)
    f = torch.ldexp(torch.ones((), dtype=torch.float64), scale.double() - 127).repeat_interleave(32, dim=-1)
    err = (back - x.double()).abs()
    assert bool((err <= torch.maximum(0.2 * x.double().abs(), 0.25 * f)).all())
    top = x.double().abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, dim=-1)
    assert bool((0.25 * f <= top / 14).all())
    assert torch.equal(back.to(torch.bfloat16).double(), back)      # bf16 holds every value
    again = quantise(back.to(torch.bfloat16))
    assert torch.equal(values(*again), back)                        # rounding what is rounded changes nothing
