"""Infinite values (scale bytes that no append stores) among the new tokens of a cache in 4 bits, where a row that sees one gives it no
weight that fp32 could hold, and rows ahead of it do not see it."""
import pytest
import torch

import mx_choice
from paged_mx_reference import MxBatch, quantise, values
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")

CASES = [      # heads, KV heads, page, by head, sequences, hints, path; a sequence is one unit, and its new tokens lie in one tile of 32 keys with the token ahead of the second
    (4, 4, 16, False, [(3, 20), (2, 50), (5, 29)], (5, 50), "units 1 8"),
    (8, 8, 32, False, [(20, 90), (28, 28), (5, 300)], (28, 300), "units 2 4"),
    (16, 2, 16, True, [(6, 95), (6, 6), (5, 230)], (6, 230), "units 3 4"),
    (8, 8, 8, False, [(3, 300), (7, 7), (2, 50)], (7, 300), "spans 1"),
    (8, 8, 16, False, [(2, 5000), (3, 90), (2, 2222), (6, 16)], (6, 5000), "spans 1"),
    (5, 1, 16, False, [(5, 9000), (2, 40), (5, 700)], (5, 9000), "spans 2"),
    (8, 1, 32, False, [(6, 9000), (6, 110), (4, 3000)], (6, 9000), "spans 3"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_%d_%d" % (c[6].replace(" ", "_"), c[0], c[2]))
@pytest.mark.parametrize("byte", [253, 254])
def test_an_infinite_value_without_weight(case, byte):
    """Every score is 0 but one of +90, of the last key that all rows see, and one of -90, of a later key whose value is infinite: 180
    apart, where fp32 holds weights down to e^-104.  The rows that see the latter get its infinities and what else there is."""
    hq, hkv, page, by_head, seqs, hints, path = case
    b = MxBatch(41, hq, hkv, page, seqs, table_extra=2)
    assert mx_choice.path(hq, hkv, seqs, hints, page, b.table.shape[1]) == path
    b.q = torch.full_like(b.q, 8.0)      # 128 dims of 8 x 1 / sqrt(128): 90.5
    for i, (n, t) in enumerate(seqs):
        size = torch.zeros(t, hkv, 128, dtype=torch.bfloat16)
        at = t - n + 1
        assert n * (hq // hkv) <= 16 * int(path.split()[1]) and (at - 1) // 32 == (t - 1) // 32
        size[at - 1], size[at] = 1.0, -1.0
        codes, scales = quantise(size)
        b.keys[i] = values(codes, scales)
        pages, slots = b.where(i)
        b.k[pages, slots], b.k_scale[pages, :, :, slots] = codes, scales
        b.v_scale[pages[at], :, 1, slots[at]] = byte
        b.v[pages[at], slots[at], :, 16:32] = torch.tensor([0xf7, 0x20], dtype=torch.uint8).repeat(8)      # 6, -6, 0, 1
        b.values[i][at, :, 32:64] = torch.tensor([INF, -INF, 0.0, 2.0 ** (byte - 127)], dtype=torch.float64).repeat(8)
    held, table, cu, len_k = b.to(DEV, by_head)
    want = attention(b)
    assert bool(want[0].isinf().any()) and not bool(want[0].isnan().any())
    for dtype in (torch.float32, torch.bfloat16):
        out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), pec.PagedCacheMx(*held), table, cu, len_k, *hints, out_dtype=dtype)
        got, inf = out.cpu().double(), want[0].isinf()
        assert not bool(got.isnan().any()), "%s: NaN in the place of an infinity" % path
        assert bool((got[inf] == want[0][inf]).all()), "%s: an infinity of the other sign" % path
        assert_attention(out, lse, want, path)
