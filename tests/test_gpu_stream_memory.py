"""Calls on the current stream and on a given one at the same time, neither with memory of its own: each result is the one of the
call alone."""
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _sync_after():
    yield
    torch.cuda.synchronize()


def two_at_once(call, here, there):
    """call(inputs, stream) on the current stream and, with other inputs of the same sizes, on another one, without a wait."""
    alone = [[t.clone() for t in call(x, None)] for x in (here, there)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(8):
        got = call(here, None), call(there, side)
        call(here, None)                       # takes over what the first one has given back on the host
        torch.cuda.synchronize()
        for results, wanted in zip(got, alone):
            for t, want in zip(results, wanted):
                assert torch.equal(t.view(torch.uint8), want.view(torch.uint8))


# the same sizes twice: steps, steps beside a list, a list in key ranges
@pytest.mark.parametrize("hints, seqs", [((8, 8000), [(1, 5000), (2, 6000), (8, 3000)]), ((300, 8000), [(300, 300), (1, 900), (8, 4000), (1, 7000)]),
                                         ((400, 8000), [(400, 5000), (1, 2000)])])
def test_paged_attention(hints, seqs):
    def inputs(seed):
        b = ref.Batch(seed, 8, 2, 16, seqs)
        kc, vc, bt, cu, lk = b.to(DEV)
        return b.q.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk

    two_at_once(lambda x, s: pec.pec_attn_paged(*x, *hints, stream=s), inputs(1), inputs(2))


def test_norm_rope_and_append():
    a = torch.arange(4000, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    turn = pec.NormRope(torch.cat([a.cos(), a.sin()], dim=1).float().to(DEV), torch.ones(128, device=DEV))

    def inputs(seed):
        b = ref.Batch(seed, 8, 2, 16, [(3000, 3000), (1, 40)])
        kc, vc, bt, cu, lk = b.to(DEV)
        kv = torch.randn(b.total, 2, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)
        return b.q.to(DEV), kv, pec.PagedCache(kc, vc), (bt, cu, lk)

    def call(x, s):
        q, kv, cache, meta = x
        qa = pec.pec_paged_append(kv, kv, cache, *meta, norm_rope=turn, q=q, stream=s)
        return (qa, *pec.pec_qk_norm_rope(q, kv, turn, stream=s))

    two_at_once(call, inputs(3), inputs(4))


def test_batches_of_keys_in_a_row():
    """pec_attn_colocated, pec_attn_varlen and pec_decode_splitkv, each with a workspace, and pec_attn_chunk."""
    lens_q, lens_k = [1, 300, 1], [9000, 2000, 4000]
    cu = [torch.tensor([0] + x, dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV) for x in (lens_q, lens_k)]

    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        return [torch.randn(n, h, 128, generator=g).to(torch.bfloat16).to(DEV) for n, h in ((sum(lens_q), 8), (sum(lens_k), 2), (sum(lens_k), 2))]

    def call(x, s):
        q, k, v = x
        return (*pec.pec_attn_colocated(q, k, v, *cu, stream=s), *pec.pec_attn_varlen(q, k[:302].contiguous(), v[:302].contiguous(), cu[0], 300, stream=s),
                *pec.pec_decode_splitkv(q[:1].contiguous(), k, v, stream=s), *pec.pec_attn_chunk(q, k, v, 14000, 0, stream=s))

    two_at_once(call, inputs(5), inputs(6))
