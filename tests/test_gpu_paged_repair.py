"""Infinite and NaN values among a chunk's own new tokens, which the rows ahead of them do not see: what such rows cost, and rows of
every kind around them."""
import pytest
import torch

import paged_reference as ref
import test_paged_infinities as inf
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# hq, hkv, page, sequences (new, all): key ranges and none, a row tile that the sequence ends in, more new tokens than tokens
@pytest.mark.parametrize("case", [(8, 2, 16, [(300, 301), (257, 6000)]), (3, 1, 8, [(500, 9000)]), (4, 4, 64, [(700, 690), (260, 1300)]),
                                  (16, 2, 32, [(400, 400), (33, 2500), (1, 900)])], ids=str)
@pytest.mark.parametrize("seed", [0, 1])
def test_values_scattered_over_the_new_tokens(case, seed):
    hq, hkv, page, seqs = case
    b = ref.Batch(70 + seed, hq, hkv, page, seqs, table_extra=inf.BIG // page)
    g = torch.Generator().manual_seed(seed)
    for i, (n, t) in enumerate(seqs):
        at = torch.randint(max(0, t - n), t, (12,), generator=g)
        for j, k in enumerate(at.tolist()):
            value = (inf.INF, -inf.INF, inf.NAN)[j % 3]
            b.values[i][k, j % hkv, int(torch.randint(0, 128, (1,), generator=g))] = value
        b.put(i)
    hints = (max(n for n, _ in seqs), inf.BIG)
    inf.check(b, hints, True, str(case))
    inf.check(b, hints, True, str(case) + " fp32", torch.float32)


def test_keys_that_are_nan_too():
    """A token whose key and value are NaN: rows that see it are, the others are as if it were not there."""
    seqs, first = [(300, 4300)], 170
    b = ref.Batch(75, 8, 2, 16, seqs, table_extra=inf.BIG // 16)
    clean = ref.attention(b)
    b.keys[0][4000 + first, 1], b.values[0][4000 + first, 1] = inf.NAN, inf.NAN
    b.put(0)
    kc, vc, bt, cu, lk = b.to(DEV)
    out, lse = pec.pec_attn_paged(b.q.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk, 300, inf.BIG)
    assert bool(out[first:, 4:].isnan().all()) and bool(lse[4:, first:].isnan().all())
    o, l = out.cpu().clone(), lse.cpu().clone()
    o[first:, 4:], l[4:, first:] = clean[0][first:, 4:].to(o.dtype), clean[1][4:, first:].float()
    ref.assert_attention(o, l, clean, "rows ahead of it")


def time_of(call):
    call()
    best = float("inf")
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


def test_one_such_value_does_not_hold_up_the_call():
    """512 new tokens behind 30,000: at most twenty times as long with a NaN in the last one's value."""
    n, t, hq, hkv, page = 512, 30512, 32, 8, 64
    g = torch.Generator(DEV).manual_seed(76)
    pages = -(-t // page)
    kc, vc = [torch.empty(pages, page, hkv, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2)]
    q = torch.empty(n, hq, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    cu, lk = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([t], dtype=torch.int32, device=DEV)
    cache = pec.PagedCache(kc, vc)
    clean = time_of(lambda: pec.pec_attn_paged(q, cache, table, cu, lk, n, t))
    vc[(t - 1) // page, (t - 1) % page, 0, 5] = inf.NAN
    odd = time_of(lambda: pec.pec_attn_paged(q, cache, table, cu, lk, n, t))
    assert odd <= 20 * clean, (odd, clean)
