"""Norms of rows whose squares fp32 holds with few bits or not at all, under an eps that does not hide them."""
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALES = [0, -40, -49, -51, -58, -62, -64, -66, -70, -76, -90, -110, -122]      # of two; bf16 has normal numbers down to 2^-126


@pytest.mark.parametrize("eps", [0.0, 1e-42, 2.0 ** -126, 2.0 ** -101, 2.0 ** -99, 1e-6])
@pytest.mark.parametrize("rotary, interleaved", [(0, False), (128, False), (64, False), (128, True)])
def test_small_rows(eps, rotary, interleaved):
    g = torch.Generator().manual_seed(7)
    scale = torch.tensor([2.0 ** s for s in SCALES], dtype=torch.float64)[:, None, None]
    x = (torch.randn(len(SCALES), 5, 128, generator=g, dtype=torch.float64) * scale).to(torch.bfloat16)
    x[2, 1] = 0
    x[3, 2, 17:] = 0
    x[5, 0] = 2.0 ** -133                      # the least number of the type
    weight = 1 + 0.3 * torch.randn(128, generator=g)
    table = None
    if rotary:
        a = torch.arange(40, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) / (rotary // 2))
        table = torch.cat([a.cos(), a.sin()], dim=1).float()
    turn = pec.NormRope(table.to(DEV) if rotary else None, q_weight=weight.to(DEV), eps=eps, interleaved=interleaved)
    got, _ = pec.pec_qk_norm_rope(x.to(DEV), None, turn)
    eps = float(torch.tensor(eps, dtype=torch.float32))      # as the call takes it: 1e-42 is 713.6 steps of 2^-149, taken as 714
    want, size = ref.norm_rope(x, weight, eps, table, torch.arange(len(SCALES)), interleaved)
    none = want.isnan()                        # a row of zeros without an eps
    assert bool(none[2, 1].all()) == (eps == 0) and int(none.sum()) == (128 if eps == 0 else 0)
    got = got.cpu()
    assert torch.equal(got.isnan(), none)
    # (below 2^-125 bf16 has steps of 2^-133: half of one more)
    size = size + 2.0 ** -134 / (80 * ref.F32)
    ref.assert_rows(torch.where(none, torch.zeros((), dtype=torch.bfloat16), got), want.masked_fill(none, 0), size.nan_to_num(0), "eps %g" % eps)
