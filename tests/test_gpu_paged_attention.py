"""pec_attn_paged against the definition in 64 bits: caches whose free slots hold NaN, pages in random order, tables that name no
page behind a sequence's last one."""
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PLAIN = pec.PEC_FLAG_SIMPLE_KERNEL


@pytest.fixture(autouse=True)
def _sync_after():
    yield
    torch.cuda.synchronize()


def run(b, causal=True, flags=0, hints=(0, 0), out_dtype=torch.bfloat16, by_head=False, q=None, **kw):
    kc, vc, bt, cu, lk = b.to(DEV, by_head)
    q = b.q.to(DEV) if q is None else q
    out = torch.full(b.q.shape, 5.0, dtype=out_dtype, device=DEV)
    lse = torch.full((b.hq, b.total), 5.0, device=DEV)
    pec.pec_attn_paged(q, pec.PagedCache(kc, vc), bt, cu, lk, max_len_q=hints[0], max_len_k=hints[1], causal=causal,
                       out_dtype=out_dtype, out=out, lse=lse, flags=flags, **kw)
    assert bool((out[b.rows:] == 5).all()) and bool((lse[:, b.rows:] == 5).all())     # rows behind the last sequence
    return out, lse


def longest(b):
    return max(n for n, _ in b.seqs), max(t for _, t in b.seqs)


# hq, hkv, page, sequences (new, all)
SMALL = [
    (1, 1, 8, [(1, 1)]),
    (4, 1, 16, [(1, 1), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 65), (1, 700)]),        # decode steps around tile ends
    (8, 8, 8, [(1, 40), (0, 30), (1, 9), (0, 0), (1, 129)]),
    (6, 2, 64, [(2, 2), (5, 100), (3, 64), (1, 128), (9, 1000)]),                                # a few new tokens, group of 3
    (10, 2, 16, [(7, 7), (7, 300), (6, 33)]),                                                    # 35 and 30 rows
    (40, 8, 32, [(1, 300), (2, 2000), (13, 13)]),
    (64, 1, 16, [(1, 500), (3, 77)]),                                                            # a group of 64
    (3, 1, 128, [(300, 300), (129, 1000), (1, 5000)]),
    (8, 2, 16, [(256, 256), (257, 400), (31, 31), (1, 2), (64, 64)]),
    (2, 2, 256, [(700, 1500)]),
    (4, 4, 16, [(3, 2), (5, 0), (4, 4), (70, 60)]),                                              # more new tokens than tokens: rows without a key
    (4, 2, 16, [(1, 1 + (37 * i) % 97) for i in range(200)]),
    (2, 1, 32, [(1 + i % 3, 5 + i) for i in range(70)] + [(100, 150)]),
]


@pytest.mark.parametrize("case", SMALL)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("flags", [0, PLAIN])
def test_small_batches(case, causal, flags):
    b = ref.Batch(len(case[3]) + case[2], *case, spare_rows=2)
    want = ref.attention(b, causal)
    for out_dtype, hints, by_head in ((torch.bfloat16, (0, 0), False), (torch.float32, longest(b), True)):
        out, lse = run(b, causal, flags, hints, out_dtype, by_head)
        ref.assert_attention(out, lse, want, "%s causal %s %s" % (case[:3], causal, out_dtype), plain=flags == PLAIN)


@pytest.mark.parametrize("hints", [(1, 1), (40, 64), (1 << 30, 1 << 30)])
def test_hints_change_no_result(hints):
    """Understated and overstated ones."""
    b = ref.Batch(3, 8, 2, 16, [(1, 900), (300, 800), (6, 50), (40, 40)])
    ref.assert_attention(*run(b, hints=hints), ref.attention(b), str(hints))


@pytest.mark.parametrize("flags", [0, PLAIN])
@pytest.mark.parametrize("seqs", [[(1, 50), (1, 300)], [(6, 90), (9, 40)], [(200, 310), (80, 80)], [(600, 700)]])
def test_what_a_row_does_not_see_does_not_reach_it(seqs, flags):
    """NaN and infinities in values and keys of later positions: rows before them are as if nothing were there."""
    for seed, (value, in_keys) in enumerate([(float("nan"), False), (float("inf"), False), (float("-inf"), False), (float("nan"), True)]):
        b = ref.Batch(60 + seed, 4, 2, 16, seqs)
        for i, (n, t) in enumerate(seqs):
            for back in {0, min(n, 3) - 1, n // 2}:                 # the last positions, n // 2 rows before the end
                (b.keys if in_keys else b.values)[i][t - 1 - back, -1, 5:9] = value
            b.put(i)
        if in_keys:      # rows that see such a key are NaN; the others are compared
            out, lse = run(b, flags=flags)
            for i, (n, t) in enumerate(seqs):
                first = min(n - 1 - back for back in {0, min(n, 3) - 1, n // 2})
                b.keys[i] = b.keys[i].nan_to_num(0.0)
                rows = slice(int(b.cu[i]), int(b.cu[i]) + first)
                want = ref.attention(b)
                part = [w[rows] if j in (0, 2) else w[:, rows] for j, w in enumerate(want)]
                ref.assert_attention(out[rows], lse[:, rows], part, "keys %s" % seqs, plain=flags == PLAIN)
                seen = slice(int(b.cu[i]) + first, int(b.cu[i + 1]))
                assert bool(out[seen, 2:].isnan().all()) and bool(lse[2:, seen].isnan().all()) and bool(out[seen, :2].isfinite().all())
        else:
            ref.assert_attention(*run(b, flags=flags), ref.attention(b), "%s %s" % (value, seqs), plain=flags == PLAIN)


@pytest.mark.parametrize("seqs", [[(1, 3000), (4, 700)], [(300, 900)]])
def test_late_jumps_of_the_row_maximum(seqs):
    """Keys that lift single rows' scores 16 ... 130 log2 units above the bulk: the softmax reference has to follow."""
    b = ref.Batch(77, 4, 2, 32, seqs)
    for i, (n, t) in enumerate(seqs):
        for key, row, gain in ((t // 3, 0, 1), (t // 2, n // 2, 2), (t - n, n - 1, 4), (t - 1, n - 1, 8), (5, 0, 3)):
            b.keys[i][key] = (b.q[int(b.cu[i]) + row, ::2].float() * gain).to(torch.bfloat16)
        b.put(i)
    for causal in (True, False):
        ref.assert_attention(*run(b, causal), ref.attention(b, causal), str(seqs))


def test_scale_strided_queries_and_shared_pages():
    b = ref.Batch(9, 8, 2, 16, [(5, 200), (1, 120), (90, 300)])
    for i in (1, 2):                                   # the first six pages of sequence 0 are a prefix of the others
        b.table[i, :6] = b.table[0, :6]
        b.keys[i][:96], b.values[i][:96] = b.keys[0][:96], b.values[0][:96]
    wide = torch.full((b.total, 12, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :8] = b.q.to(DEV)
    out, lse = run(b, q=wide[:, :8], scale=0.03)
    ref.assert_attention(out, lse, ref.attention(b, scale=0.03), "strided")


def test_no_sequence_and_no_row():
    b = ref.Batch(11, 4, 2, 16, [(0, 40), (0, 0)], spare_rows=5)
    run(b)
    b = ref.Batch(12, 4, 2, 16, [(2, 0), (1, 0)], table_extra=0)       # a table without a column
    out, lse = run(b)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("flags", [0, PLAIN])
def test_offsets_past_four_gigabytes(flags):
    """Pages at the far end of a cache of more than 2^32 bytes and 2^31 elements, in K and in V."""
    page, hkv, n_pages = 64, 8, 20000                  # 2.6 GB per 20000 pages x 131,072 bytes each
    kc = torch.zeros(n_pages * 2, page, hkv, 128, dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    b = ref.Batch(13, 8, 8, page, [(1, 200), (2, 150), (70, 300)], wild=False)
    far = torch.tensor([0] + [n_pages * 2 - 1 - i for i in range(b.n_pages - 1)])
    assert int(far.max()) * page * hkv * 128 > 2 ** 31
    kc[far.to(DEV)], vc[far.to(DEV)] = b.k.to(DEV), b.v.to(DEV)
    table = far.to(torch.int32)[b.table.long()].to(DEV)
    want = ref.attention(b)
    out, lse = pec.pec_attn_paged(b.q.to(DEV), pec.PagedCache(kc, vc), table, b.cu.to(DEV), b.len_k.to(DEV), flags=flags)
    ref.assert_attention(out, lse, want, "far pages", plain=flags == PLAIN)


def test_malformed_batches_stay_in_bounds():
    """Offsets that fall, lengths beyond the table, page numbers outside the cache: some result, nothing out of bounds, and the
    rows of no sequence left alone."""
    b = ref.Batch(14, 4, 2, 16, [(3, 50), (40, 90), (1, 20)], spare_rows=4)
    b.cu = torch.tensor([0, 46, 43, 44], dtype=torch.int32)
    b.len_k = torch.tensor([2 ** 31 - 1, -7, 1000], dtype=torch.int32)
    kc, vc, bt, cu, lk = b.to(DEV)
    for flags in (0, PLAIN):
        for hints in ((0, 0), (1, 64)):
            out = torch.full(b.q.shape, 5.0, dtype=torch.bfloat16, device=DEV)
            lse = torch.full((4, b.total), 5.0, device=DEV)
            pec.pec_attn_paged(b.q.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk, *hints, out=out, lse=lse, flags=flags)
            torch.cuda.synchronize()
            assert bool((out[47:] == 5).all()) and bool((lse[:, 47:] == 5).all())
