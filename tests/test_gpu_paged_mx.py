"""The paged cache in 4 bits on the GPU: what is stored, what is read back, attention over it."""
import math

import pytest
import torch

import mx_choice
from paged_mx_reference import MxBatch, quantise, values
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"

SEQS = {
    "one token": [(1, 1)],
    "steps": [(1, 37), (1, 1), (1, 64), (1, 500), (1, 16)],
    "drafted": [(5, 129), (3, 3), (4, 77)],
    "chunks": [(70, 70), (33, 200), (1, 90), (0, 40), (129, 130)],
    "empty": [(0, 0), (2, 9), (0, 0)],
}


def caches(batch, by_head=False):
    held, table, cu, len_k = batch.to(DEV, by_head)
    return pec.PagedCacheMx(*held), table, cu, len_k


def rows_of(batch, new_only=True):
    """(page, slot) of every packed row, and the tokens' keys and values before rounding."""
    pages, slots, k, v = [], [], [], []
    for b, (n, t) in enumerate(batch.seqs):
        p, s = batch.where(b, t - n if new_only else 0)
        pages.append(p)
        slots.append(s)
        k.append(batch.raw[b][0][t - n:])
        v.append(batch.raw[b][1][t - n:])
    return torch.cat(pages), torch.cat(slots), torch.cat(k), torch.cat(v)


@pytest.mark.parametrize("hkv,page,by_head", [(1, 8, False), (2, 16, False), (5, 16, True), (8, 64, False)])
@pytest.mark.parametrize("seqs", list(SEQS), ids=lambda s: s.replace(" ", "_"))
def test_append_and_read(seqs, hkv, page, by_head):
    """Codes and scales bit for bit, nothing else touched; what comes back is what they stand for."""
    b = MxBatch(3, 2 * hkv, hkv, page, SEQS[seqs], spare_rows=3)
    pages, slots, k, v = rows_of(b)
    g = torch.Generator().manual_seed(9)
    size = torch.exp(4 * torch.randn(k.shape[0], hkv, 4, 1, generator=g)).repeat_interleave(32, dim=2).flatten(-2)
    k, v = (k.float() * size).to(torch.bfloat16), (v.float() * size.flip(0)).to(torch.bfloat16)
    cache, table, cu, len_k = caches(b, by_head)
    want = [t.clone() for t in (b.k, b.v, b.k_scale, b.v_scale)]
    for x, c, s in ((k, want[0], want[2]), (v, want[1], want[3])):
        c[pages, slots], s[pages, :, :, slots] = quantise(x)
    qkv = torch.randn(b.total, 4 * hkv, 128, generator=g).to(torch.bfloat16)
    qkv[:b.rows, 2 * hkv:3 * hkv], qkv[:b.rows, 3 * hkv:] = k, v
    d = qkv.to(DEV)
    kd, vd = d[:, 2 * hkv:3 * hkv], d[:, 3 * hkv:]
    pec.pec_paged_append_mx(kd, vd, cache, table, cu, len_k)
    for got, ref, name in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want, ("k", "v", "k_scale", "v_scale")):
        assert torch.equal(got.cpu(), ref), name
    ko, vo = [torch.full((b.total, hkv, 128), 77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pec.pec_paged_read_mx(cache, table, cu, len_k, k=ko, v=vo)
    for got, c, s in ((ko, want[0], want[2]), (vo, want[1], want[3])):
        assert torch.equal(got[:b.rows].cpu().double(), values(c[pages, slots], s[pages, :, :, slots]))
        assert bool((got[b.rows:] == 77).all())


def test_read_whole_sequences():
    b = MxBatch(4, 4, 2, 16, [(1, 300), (3, 17), (0, 5)])
    cache, table, cu, len_k = caches(b)
    cu = torch.cumsum(torch.tensor([0] + [t for _, t in b.seqs]), 0).to(torch.int32).to(DEV)
    k, v = pec.pec_paged_read_mx(cache, table, cu, len_k, total_q=322)
    assert torch.equal(k.cpu().double(), torch.cat(b.keys)) and torch.equal(v.cpu().double(), torch.cat(b.values))


def special_rows():
    """Head rows with zeros, signed zeros, ties, the largest and smallest numbers, infinities and NaN in one group."""
    inf, nan, big = math.inf, math.nan, 3.3895313892515355e38
    heads = [[0.0], [-0.0, 0.0], [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0], [7.0, 3.5, 0.5], [6.96875, -7.0],
             [big, -big, big / 3], [2.0 ** 127, 1.0], [2.0 ** -126, -(2.0 ** -127), 2.0 ** -133], [2.0 ** -133], [1e-30, 3e-30, 1.1e-30],
             [inf, 1.0], [1.0, -inf], [nan], [1.0, nan, inf], [1.0] * 32, [-448.0, 447.0]]
    x = torch.zeros(len(heads), 1, 128, dtype=torch.bfloat16)
    for i, h in enumerate(heads):
        for g in range(4):
            at = 32 * g if g != 1 else 32 * g + 32 - len(h)
            x[i, 0, at:at + len(h)] = torch.tensor(h, dtype=torch.bfloat16) if g < 3 else 0.5
    return x


def test_append_special_values():
    x = special_rows()
    n = x.shape[0]
    b = MxBatch(5, 1, 1, 16, [(n, n)])
    cache, table, cu, len_k = caches(b)
    pec.pec_paged_append_mx(x.to(DEV), x.flip(0).contiguous().to(DEV), cache, table, cu, len_k)
    pages, slots = b.where(0)
    for codes, scales, ref in ((cache.k, cache.k_scale, x), (cache.v, cache.v_scale, x.flip(0))):
        c, s = quantise(ref)
        assert torch.equal(scales.cpu()[pages, :, :, slots], s)
        assert torch.equal(codes.cpu()[pages, slots], c)
    k, _ = pec.pec_paged_read_mx(cache, table, cu, len_k, total_q=n)
    want = values(*quantise(x))
    assert torch.equal(k.cpu().double().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm,rotary", [(False, 0), (True, 0), (False, 128), (True, 128), (True, 64)])
def test_append_norms_and_rotates_as_the_cache_of_bf16(norm, rotary, interleaved):
    """The codes are those of the very rows that pec_paged_append stores, and the queries are the same."""
    b = MxBatch(6, 9, 3, 16, [(40, 90), (1, 33), (7, 7)], spare_rows=1)
    cache, table, cu, len_k = caches(b)
    g = torch.Generator().manual_seed(2)
    rnd = lambda h: torch.randn(b.total, h, 128, generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    q, k, v = rnd(9), rnd(3), rnd(3)
    angle = torch.randn(90, max(rotary // 2, 1), generator=g)
    table_cs = torch.cat([angle.cos(), angle.sin()], dim=1).to(DEV) if rotary else None
    w = [1 + 0.3 * torch.randn(128, generator=g).to(DEV) for _ in range(2)] if norm else [None, None]
    turn = pec.NormRope(table_cs, w[0], w[1], interleaved=interleaved)
    plain = pec.PagedCache(*[torch.zeros(b.n_pages, 16, 3, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)])
    ref_q, got_q = torch.zeros_like(q), torch.zeros_like(q)
    pec.pec_paged_append(k, v, plain, table, cu, len_k, norm_rope=turn, q=q, q_out=ref_q)
    pec.pec_paged_append_mx(k, v, cache, table, cu, len_k, norm_rope=turn, q=q, q_out=got_q)
    assert torch.equal(ref_q, got_q)
    for i in range(3):
        page, slot = b.where(i, b.seqs[i][1] - b.seqs[i][0])
        for held, codes, scales in ((plain.k, cache.k, cache.k_scale), (plain.v, cache.v, cache.v_scale)):
            c, s = quantise(held.cpu()[page, slot])
            assert torch.equal(codes.cpu()[page, slot], c) and torch.equal(scales.cpu()[page, :, :, slot], s)


def test_tokens_without_a_place():
    """Positions before 0, behind the table's row and pages outside the cache: not stored, read as zeros."""
    hkv, page = 2, 8
    z = lambda *s: torch.full(s, 9, dtype=torch.uint8, device=DEV)  # noqa: E731
    cache = pec.PagedCacheMx(z(3, page, hkv, 64), z(3, page, hkv, 64), z(3, hkv, 4, page), z(3, hkv, 4, page))
    table = torch.tensor([[0, 7], [-1, 1], [2, 2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 4, 8, 12], dtype=torch.int32, device=DEV)
    len_k = torch.tensor([2, 18, 10], dtype=torch.int32, device=DEV)      # positions -2 ... 1; 12 ... 15 (18 is cut to 16); 6 ... 9
    x = torch.ones(12, hkv, 128, dtype=torch.bfloat16, device=DEV)
    pec.pec_paged_append_mx(x, x, cache, table, cu, len_k)
    k, v = pec.pec_paged_read_mx(cache, table, cu, len_k, total_q=12)
    stored = [False, False, True, True, True, True, True, True, True, True, False, False]
    assert (k[:, 0, 0] == 1).tolist() == stored and (v[:, 1, 77] == 1).tolist() == stored
    assert bool((k[~torch.tensor(stored, device=DEV)] == 0).all())
    touched = (cache.k_scale != 9).any(dim=2)[:, 0].cpu()
    assert touched.sum() == 8 and touched[0, :2].all() and touched[1, 4:].all() and touched[2, 6:].all()


@pytest.mark.parametrize("flags", [pec.PEC_FLAG_SIMPLE_KERNEL, 0], ids=["simple", "fast"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,page,by_head", [(4, 4, 8, False), (8, 2, 16, True), (5, 1, 64, False), (16, 2, 32, False), (40, 2, 16, False)])
@pytest.mark.parametrize("seqs", list(SEQS), ids=lambda s: s.replace(" ", "_"))
def test_attention(seqs, hq, hkv, page, by_head, causal, flags):
    b = MxBatch(11, hq, hkv, page, SEQS[seqs], spare_rows=2)
    cache, table, cu, len_k = caches(b, by_head)
    ref = attention(b, causal)
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((b.total, hq, 128), 55.0, dtype=dtype, device=DEV)
        lse = torch.full((hq, b.total), 55.0, device=DEV)
        pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, causal=causal, out_dtype=dtype, flags=flags, out=out, lse=lse)
        assert_attention(out, lse, ref, "%s %s" % (seqs, dtype), plain=flags != 0)
        assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


@pytest.mark.parametrize("hints", [True, False])
@pytest.mark.parametrize("hq,hkv,page", [(8, 2, 16), (16, 16, 8), (6, 1, 128)])
def test_chunks_beside_steps(hq, hkv, page, hints):
    """Sequences with few rows and sequences with many are launched apart, each with their own cut."""
    seqs = [(1, 190), (70, 70), (150, 400), (1, 5), (0, 90), (40, 64), (1, 1), (300, 301), (1, 700), (2, 30), (17, 17)]
    b = MxBatch(13, hq, hkv, page, seqs, spare_rows=2, table_extra=20000 // page)
    cache, table, cu, len_k = caches(b)
    ref = attention(b)
    assert mx_choice.path(hq, hkv, seqs, (300, 700) if hints else (0, 0), page, table.shape[1], 2, True) == "beside"
    ws = torch.full((pec.pec_paged_mx_workspace_bytes(hq, hkv, len(seqs), b.total),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((b.total, hq, 128), 55.0, dtype=torch.float32, device=DEV)
    lse = torch.full((hq, b.total), 55.0, device=DEV)
    pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, max_len_q=300 if hints else 0, max_len_k=700 if hints else 0,
                          out_dtype=torch.float32, out=out, lse=lse, workspace=ws)
    assert_attention(out, lse, ref)
    assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


@pytest.mark.parametrize("room", [0, 520, 1400, 3000, 100000])
def test_chunks_with_room_for_some(room):
    """Keys of sequences in bf16 as far as the workspace goes; all of them give the same."""
    seqs = [(500, 500), (400, 900), (300, 300)]
    b = MxBatch(13, 32, 8, 64, seqs, spare_rows=2, table_extra=600)
    cache, table, cu, len_k = caches(b)
    assert mx_choice.path(32, 8, seqs, (512, 30512), 64, table.shape[1], 2, True) == "list"
    ws = torch.full((pec.pec_paged_mx_workspace_bytes(32, 8, len(seqs), b.total, room),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((b.total, 32, 128), 55.0, dtype=torch.float32, device=DEV)
    lse = torch.full((32, b.total), 55.0, device=DEV)
    pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, max_len_q=512, max_len_k=30512, out_dtype=torch.float32, out=out, lse=lse,
                          workspace=ws)
    assert_attention(out, lse, attention(b))
    assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


@pytest.mark.parametrize("room", [0, 1500, 100000])
@pytest.mark.parametrize("causal", [True, False])
def test_one_chunk(causal, room):
    b = MxBatch(14, 8, 2, 32, [(333, 1500)])
    cache, table, cu, len_k = caches(b)
    table = table[:, :47].contiguous()      # no wider than the sequence: then all of it has room for certain
    ws = torch.full((pec.pec_paged_mx_workspace_bytes(8, 2, 1, b.total, room),), 0xff, dtype=torch.uint8, device=DEV)
    out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, causal=causal, workspace=ws)
    assert_attention(out, lse, attention(b, causal))


def test_two_tokens_for_one_slot():
    """Sequences that share a page: its slots hold bytes of one or the other, and nothing else changes."""
    hkv = 2
    b = MxBatch(6, 4, hkv, 16, [(3, 19), (3, 19), (2, 8)])
    b.table[1, 1] = b.table[0, 1]                # positions 16, 17, 18 of both
    pages, slots, k, v = rows_of(b)
    cache, table, cu, len_k = caches(b)
    pec.pec_paged_append_mx(k.to(DEV), v.to(DEV), cache, table, cu, len_k)
    for got_c, got_s, c, s, x in ((cache.k, cache.k_scale, b.k, b.k_scale, k), (cache.v, cache.v_scale, b.v, b.v_scale, v)):
        got_c, got_s, (codes, scales) = got_c.cpu(), got_s.cpu(), quantise(x)
        for i in range(3):
            at = (pages[i], slots[i])
            assert bool(((got_c[at] == codes[i]) | (got_c[at] == codes[3 + i])).all())
            mine = got_s[at[0], :, :, at[1]]
            assert bool(((mine == scales[i]) | (mine == scales[3 + i])).all())
        want_c, want_s = c.clone(), s.clone()
        want_c[pages, slots], want_s[pages, :, :, slots] = codes, scales
        want_c[pages[:3], slots[:3]], want_s[pages[:3], :, :, slots[:3]] = got_c[pages[:3], slots[:3]], got_s[pages[:3], :, :, slots[:3]]
        assert torch.equal(got_c, want_c) and torch.equal(got_s, want_s)
