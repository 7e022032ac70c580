"""Every code with every scale byte, read back; and more KV heads than a workgroup takes side by side."""
import pytest
import torch

import mx_choice
from paged_mx_reference import MxBatch, values
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("page,by_head", [(8, False), (64, True)])
def test_every_code_with_every_scale_byte(page, by_head):
    """What the codes stand for, rounded to bf16 where that has no such number: byte 0 gives 2^-127, 253 and 254 infinities, 255 NaN."""
    n, hkv = 256, 2
    cu, len_k = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    byte = torch.arange(n, dtype=torch.uint8)
    pair = torch.arange(256, dtype=torch.uint8).view(1, 4, 64)      # all pairs of codes in four rows of 64 bytes
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(3)).to(torch.int32)[None]
    for part in range(4):
        codes = torch.stack([pair[:, part], pair[:, part].flip(-1)], dim=1).expand(n, hkv, 64).contiguous()
        scale = torch.stack([byte.roll(64 * g) for g in range(4)], dim=-1)[:, None].expand(n, hkv, 4).contiguous()
        shape = (n // page, hkv, page, 64) if by_head else (n // page, page, hkv, 64)
        held = [torch.zeros(shape, dtype=torch.uint8) for _ in range(2)]
        held = [t.transpose(1, 2) if by_head else t for t in held]
        scales = [torch.zeros(n // page, hkv, 4, page, dtype=torch.uint8) for _ in range(2)]
        pos = torch.arange(n)
        where = table[0].long()[pos // page], pos % page
        for t, s in zip(held, scales):
            t[where] = codes
            s[where[0], :, :, where[1]] = scale
        held = [t.transpose(1, 2).to(DEV).transpose(1, 2) if by_head else t.to(DEV) for t in held]
        cache = pec.PagedCacheMx(*held, *[s.to(DEV) for s in scales])
        want = values(codes, scale).to(torch.float32).to(torch.bfloat16)      # (2^129 and more are beyond fp32, too)
        for got in pec.pec_paged_read_mx(cache, table.to(DEV), cu, len_k, total_q=n):
            assert torch.equal(got.cpu().double().nan_to_num(nan=12345.0), want.double().nan_to_num(nan=12345.0))
            assert torch.equal(torch.signbit(got.cpu())[~want.isnan()], torch.signbit(want)[~want.isnan()])


@pytest.mark.parametrize("hkv", [16, 24])
def test_decode_steps_of_many_kv_heads_by_token(hkv):
    seqs = [(1, 5000), (1, 90), (1, 2222), (0, 30), (1, 16)]
    b = MxBatch(42, hkv, hkv, 16, seqs, spare_rows=1)
    assert mx_choice.path(hkv, hkv, seqs, (1, 5000), 16, b.table.shape[1], 1) == "spans 1"
    held, table, cu, len_k = b.to(DEV)
    for causal in (True, False):
        out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), pec.PagedCacheMx(*held), table, cu, len_k, 1, 5000, causal=causal, out_dtype=torch.float32)
        assert_attention(out, lse, attention(b, causal))
