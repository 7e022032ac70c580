"""pec_qk_norm_rope and pec_paged_append against the definitions in 64 bits."""
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


@pytest.fixture(autouse=True)
def _sync_after():
    yield
    torch.cuda.synchronize()


def angles(n, rotary):
    half = rotary // 2
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def made(seed, norm, rotary, interleaved, n_pos):
    g = torch.Generator().manual_seed(seed)
    qw, kw = [1 + 0.3 * torch.randn(128, generator=g) if norm else None for _ in range(2)]
    table = angles(n_pos, rotary) if rotary else None
    on = [t.to(DEV) if t is not None else None for t in (table, qw, kw)]
    return table, qw, kw, pec.NormRope(*on, eps=EPS, interleaved=interleaved)


# tokens, hq, hkv, norm, rotary, interleaved, packed
ROPE = [(1, 1, 1, True, 128, False, False), (5, 6, 2, True, 128, False, True), (7, 3, 1, False, 128, True, True),
        (64, 32, 8, True, 128, True, True), (33, 5, 5, True, 48, False, True), (33, 8, 4, False, 16, True, False),
        (130, 12, 3, False, 96, False, True), (2050, 8, 8, True, 64, False, True), (5000, 10, 2, True, 128, False, False),
        (300, 7, 7, True, 0, False, True), (20, 64, 8, True, 112, True, True), (3, 40, 1, False, 0, False, True)]


@pytest.mark.parametrize("case", ROPE)
@pytest.mark.parametrize("how", ["own positions", "pos0", "in place"])
def test_norm_rope(case, how):
    tokens, hq, hkv, norm, rotary, interleaved, packed = case
    n_pos = 9000
    table, qw, kw, handle = made(tokens, norm, rotary, interleaved, n_pos)
    g = torch.Generator().manual_seed(tokens + 1)
    scale = torch.exp2(torch.randint(-8, 9, (tokens, 1, 1), generator=g).float())
    qkv = (torch.randn(tokens, hq + 2 * hkv, 128, generator=g) * scale).to(torch.bfloat16)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    dev = qkv.to(DEV)
    dq, dk = dev[:, :hq], dev[:, hq:hq + hkv]
    if not packed or how == "in place":
        dq, dk = dq.contiguous(), dk.contiguous()
    at = torch.randint(0, n_pos, (tokens,), generator=g, dtype=torch.int32)
    kw_args = {"positions": at.to(DEV)}
    if how == "pos0":
        at, kw_args = torch.arange(17, 17 + tokens), {"pos0": 17}
    if how == "in place":
        kw_args.update(q_out=dq, k_out=dk)
    qo, ko = pec.pec_qk_norm_rope(dq, dk, handle, **kw_args)
    for got, x, w, what in ((qo, q, qw, "q"), (ko, k, kw, "k")):
        ref.assert_rows(got, *ref.norm_rope(x, w, EPS, table, at, interleaved), "%s of %s" % (what, case))


def test_queries_or_keys_alone_and_one_weight():
    table, qw, kw, handle = made(3, True, 128, False, 100)
    x = torch.randn(9, 6, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    at = torch.arange(9) + 20
    qo, none = pec.pec_qk_norm_rope(x.to(DEV), None, handle, pos0=20)
    none2, ko = pec.pec_qk_norm_rope(None, x.to(DEV), handle, pos0=20)
    assert none is None and none2 is None
    ref.assert_rows(qo, *ref.norm_rope(x, qw, EPS, table, at), "q")
    ref.assert_rows(ko, *ref.norm_rope(x, kw, EPS, table, at), "k")
    only_q = pec.NormRope(table.to(DEV), q_weight=qw.to(DEV), eps=EPS)
    qo, ko = pec.pec_qk_norm_rope(x.to(DEV), x.to(DEV), only_q, pos0=20)
    ref.assert_rows(qo, *ref.norm_rope(x, qw, EPS, table, at), "q with a weight")
    ref.assert_rows(ko, *ref.norm_rope(x, None, EPS, table, at), "k without")


def test_rows_of_zeros_of_large_values_and_of_nan_keep_to_themselves():
    table, qw, kw, handle = made(5, True, 64, False, 100)
    x = torch.randn(12, 4, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    x[3] = 0
    x[5, 2] = float("nan")
    x[6, 1, 100] = float("inf")
    x[7] *= 2.0 ** 50                       # squares that fp32 holds
    plain = pec.NormRope(table.to(DEV))
    for h, w in ((handle, qw), (plain, None)):
        qo, _ = pec.pec_qk_norm_rope(x.to(DEV), None, h, pos0=0)
        want, size = ref.norm_rope(x, w, EPS, table, torch.arange(12))
        fine = want.isfinite()
        assert torch.equal(qo.cpu().isfinite(), fine)
        ref.assert_rows(torch.where(fine, qo.cpu(), torch.zeros((), dtype=torch.bfloat16)), want.masked_fill(~fine, 0), size.nan_to_num(0, 0, 0))


def test_positions_outside_the_table_are_taken_at_its_ends():
    table, _, _, handle = made(7, False, 128, False, 50)
    x = torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    at = torch.tensor([-3, 49, 50, 2 ** 31 - 1], dtype=torch.int32)
    qo, _ = pec.pec_qk_norm_rope(x.to(DEV), None, handle, positions=at.to(DEV))
    ref.assert_rows(qo, *ref.norm_rope(x, None, EPS, table, at))


# hq, hkv, page, sequences (new, all), norm, rotary, interleaved, by_head
APPEND = [(8, 2, 16, [(1, 1), (1, 17), (1, 16), (1, 300)], True, 128, False, False),
          (4, 4, 8, [(5, 5), (0, 9), (3, 40), (1, 8), (0, 0)], False, 64, True, True),
          (6, 1, 64, [(200, 1000), (1, 64), (129, 129)], True, 128, False, True),
          (3, 3, 32, [(70, 70)], False, 0, False, False),
          (32, 8, 256, [(1, n) for n in range(1, 150)], True, 128, True, False),
          (2, 1, 16, [(1, 1 + n % 40) for n in range(4500)], False, 128, False, False),
          (5, 5, 16, [(0, 5)] * 70 + [(4, 9)] + [(0, 3)] * 70 + [(2, 2)], True, 48, False, False)]


@pytest.mark.parametrize("case", APPEND)
def test_append(case):
    hq, hkv, page, seqs, norm, rotary, interleaved, by_head = case
    b = ref.Batch(90 + page + len(seqs), hq, hkv, page, seqs, spare_rows=3)
    table, qw, kw, handle = made(page, norm, rotary, interleaved, 1 + max(t for _, t in seqs))
    new = torch.randn(b.total, hq + 2 * hkv, 128, generator=torch.Generator().manual_seed(page)).to(torch.bfloat16)
    at = torch.cat([torch.arange(t - n, t) for n, t in seqs])
    owner = torch.cat([torch.full((n,), i) for i, (n, _) in enumerate(seqs)])
    kc, vc, bt, cu, lk = b.to(DEV, by_head)
    cache = pec.PagedCache(kc, vc)
    dev = new.to(DEV)
    q_out = torch.full((b.total, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    got = pec.pec_paged_append(dev[:, hq:hq + hkv], dev[:, hq + hkv:], cache, bt, cu, lk, norm_rope=handle, q=dev[:, :hq], q_out=q_out)
    assert got is q_out and bool((q_out[b.rows:] == 7).all())        # rows behind the last sequence
    n = b.rows
    ref.assert_rows(q_out[:n], *ref.norm_rope(new[:n, :hq], qw, EPS, table, at, interleaved), "q")
    where = b.table.long()[owner, at // page], at % page
    ref.assert_rows(kc.cpu()[where], *ref.norm_rope(new[:n, hq:hq + hkv], kw, EPS, table, at, interleaved), "k")
    assert torch.equal(vc.cpu()[where].view(torch.int16), new[:n, hq + hkv:].view(torch.int16))
    for mine, before in ((kc, b.k), (vc, b.v)):                      # every other slot as it was, NaN bits and all
        mine, before = mine.cpu().clone(), before.clone()
        mine[where] = before[where] = 0
        assert torch.equal(mine.view(torch.int16), before.view(torch.int16))


def test_append_without_norm_rope_copies_bits_and_leaves_queries_out():
    b = ref.Batch(5, 4, 2, 16, [(3, 20), (1, 1)])
    kc, vc, bt, cu, lk = b.to(DEV)
    new = torch.randn(b.total, 4, 128).to(torch.bfloat16)
    new[1, 0, 3] = float("nan")
    dev = new.to(DEV)
    assert pec.pec_paged_append(dev[:, :2], dev[:, 2:], pec.PagedCache(kc, vc), bt, cu, lk) is None
    for i, (s, p) in enumerate([(0, 17), (0, 18), (0, 19), (1, 0)]):
        page, slot = int(b.table[s, p // 16]), p % 16
        assert torch.equal(kc[page, slot].cpu().view(torch.int16), new[i, :2].view(torch.int16))
        assert torch.equal(vc[page, slot].cpu().view(torch.int16), new[i, 2:].view(torch.int16))


def test_append_stores_nothing_for_tokens_without_a_place():
    """Negative positions, positions behind the table's row, page numbers outside the cache, offsets that fall."""
    b = ref.Batch(6, 2, 2, 16, [(4, 2), (2, 16), (3, 40), (2, 30)], table_extra=0)
    b.table[3, 1] = b.n_pages                       # a page that does not exist, for position 28, 29
    b.len_k[2] = 16 * b.table.shape[1] + 100        # clamped to what the row holds: its last three slots
    kc, vc, bt, cu, lk = b.to(DEV)
    new = torch.randn(b.total, 4, 128).to(torch.bfloat16).to(DEV)
    q = torch.randn(b.total, 2, 128).to(torch.bfloat16).to(DEV)
    out = pec.pec_paged_append(new[:, :2], new[:, 2:], pec.PagedCache(kc, vc), bt, cu, lk, q=q)
    assert torch.equal(out, q)
    placed = [(2, 0, 0), (3, 0, 1), (4, 1, 14), (5, 1, 15)] + [(6 + i, 2, 16 * b.table.shape[1] - 3 + i) for i in range(3)]
    want = b.k.clone()
    for row, s, p in placed:
        number = int(b.table[s, p // 16])
        if 0 <= number < b.n_pages:
            want[number, p % 16] = new[row, :2].cpu()
    assert torch.equal(kc.cpu().view(torch.int16), want.view(torch.int16))
    cu = torch.tensor([0, 500, -3, 7, 2], dtype=torch.int32, device=DEV)
    pec.pec_paged_append(new[:, :2], new[:, 2:], pec.PagedCache(kc, vc), bt, cu, lk, q=q)      # stays in bounds
