"""How far a value is from what a cache in 4 bits holds of it, over every bf16 number as a group's largest, with the scales' ends."""
import torch

from paged_mx_reference import quantise, values


def groups():
    """(rows [n, 128] bf16: in every group its largest and 31 others up to it, the group's largest [n, 4])"""
    top = torch.arange(1, 0x7f80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(8)
    part = torch.rand(top.numel(), 31, generator=g, dtype=torch.float64)
    part[::2] *= part[::2] * part[::2]
    other = (part * top.double()[:, None]).to(torch.bfloat16)
    other = torch.minimum(other, top[:, None]) * torch.where(torch.rand(other.shape, generator=g) < 0.5, -1.0, 1.0).to(torch.bfloat16)
    group = torch.cat([top[:, None], other], dim=1)
    pad = -group.shape[0] % 4
    group = torch.cat([group, torch.ones(pad, 32, dtype=torch.bfloat16)])
    return group.view(-1, 128), group.abs().amax(dim=1).double()


def test_the_bound_of_the_header():
    x, top = groups()
    codes, scale = quantise(x)
    err = (values(codes, scale) - x.double()).abs().view(-1, 32)
    x = x.double().abs().view(-1, 32)
    f = torch.ldexp(torch.ones((), dtype=torch.float64), scale.double().flatten() - 127)[:, None]
    within = (top >= 3.5 * 2.0 ** -125) & (top < 7 * 2.0 ** 125)
    assert within.sum() > 31000 and (f[within] <= top[within, None] / 3.5).all()      # 0.25 x scale: 1/14 of the largest
    assert (err[within] <= torch.maximum(0.2 * x, 0.25 * f)[within]).all()
    small, large = top < 3.5 * 2.0 ** -125, top >= 7 * 2.0 ** 125
    assert (f[small] == 2.0 ** -125).all() and (err[small] <= torch.clamp(0.2 * x, min=2.0 ** -127)[small]).all()
    assert (f[large] == 2.0 ** 125).all() and (err[large] <= torch.maximum(0.25 * x, 0.25 * f)[large]).all()
    # and it does not hold there
    assert (0.25 * f[small] > top[small, None] / 14).any() and (err[large] > torch.maximum(0.2 * x, 0.25 * f)[large]).any()
