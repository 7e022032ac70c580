"""Norms, rotation and append of more tokens than one dimension of a launch has threads for (2^32 of them, a wavefront per token)."""
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOKENS = (1 << 26) + 3          # 17 GB of one head


@pytest.fixture(autouse=True)
def _free_after():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def looked_at():
    g = torch.Generator().manual_seed(1)
    some = torch.randint(0, TOKENS, (200,), generator=g)
    return torch.cat([torch.arange(9), torch.arange(TOKENS - 20, TOKENS), some]).unique()


def test_norm_rope():
    x = torch.empty(TOKENS, 1, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(2))
    at = looked_at()
    before = x[at.to(DEV)].cpu()
    weight = 1 + 0.2 * torch.randn(128, generator=torch.Generator().manual_seed(3))
    pec.pec_qk_norm_rope(x, None, pec.NormRope(q_weight=weight.to(DEV)), q_out=x)
    ref.assert_rows(x[at.to(DEV)], *ref.norm_rope(before, weight, 1e-6), "in place")


def test_append():
    x = torch.empty(TOKENS, 1, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(4))
    pages = -(-TOKENS // 256)
    kc = torch.zeros(pages, 256, 1, 128, dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(5)).to(torch.int32)
    n = torch.tensor([TOKENS], dtype=torch.int32, device=DEV)
    pec.pec_paged_append(x, x, pec.PagedCache(kc, vc), table[None].to(DEV), torch.tensor([0, TOKENS], dtype=torch.int32, device=DEV), n)
    at = looked_at()
    where = table.long()[at // 256].to(DEV), (at % 256).to(DEV)
    want = x[at.to(DEV)].view(torch.int16)
    assert bool((kc[where].view(torch.int16) == want).all()) and bool((vc[where].view(torch.int16) == want).all())


# (the hints choose units: tests/test_many_tokens_path.py)
SEQUENCES, HEADS, HINTS, TABLE = 16384, 1024, (300, 3000), 400


def test_attention_of_many_heads():
    """A workgroup for every sequence and KV head, 17 million of them: a sequence of one token gets its value and its score."""
    g = torch.Generator(DEV).manual_seed(6)
    pages = 64
    kc, vc = [torch.empty(pages, 8, HEADS, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2)]
    q = torch.empty(SEQUENCES, HEADS, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    table = torch.full((SEQUENCES, TABLE), -1, dtype=torch.int32, device=DEV)
    table[:, 0] = torch.randint(0, pages, (SEQUENCES,), generator=g, device=DEV, dtype=torch.int32)
    cu = torch.arange(SEQUENCES + 1, dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0)
    lse = torch.full((HEADS, SEQUENCES), 7.0, device=DEV)
    pec.pec_attn_paged(q, pec.PagedCache(kc, vc), table, cu, torch.ones(SEQUENCES, dtype=torch.int32, device=DEV), *HINTS, out=out, lse=lse)
    for r in range(0, SEQUENCES, 2048):
        number = table[r:r + 2048, 0].long()
        assert bool((out[r:r + 2048].view(torch.int16) == vc[number, 0].view(torch.int16)).all())
        product = q[r:r + 2048].double() * kc[number, 0].double() * 128 ** -0.5
        want = product.sum(dim=-1).T
        allowed = 2 * (128 * ref.F32 * product.abs().sum(dim=-1).T + 2.0 ** -20) + 2.0 ** -20 * want.abs()
        assert bool(((lse[:, r:r + 2048].double() - want).abs() <= allowed).all())
