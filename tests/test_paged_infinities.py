"""Infinite and NaN values of keys that a row does see: every way in which a call is cut gives the definition's infinity, its sign,
or NaN, whatever the length that the sequence has behind its last whole tile."""
import pytest
import torch

import paged_choice as choice
import paged_reference as ref
from paper_2409_15104_amd import binding as pec

DEV = "cuda:0"
BIG = 8000      # keys that every block table here has room for
INF, NAN = float("inf"), float("nan")
# path, hq, hkv, sequences (new, all), hints.  Tiles are of 32 or 64 keys and wavefronts of 32 rows: lengths behind a tile's end by 1
# and up to 63, at it, and last wavefronts with one row and with more
SEQS = [(33, 65), (65, 129), (1, 100), (97, 127), (64, 128), (40, 191), (1, 1), (2, 33)]
PATHS = [
    ("units 8", 4, 2, SEQS, (97, 191)),
    ("steps 1", 4, 2, [(1, 65), (2, 129), (16, 100), (1, 64), (3, 7000)], (16, BIG)),
    ("steps 2", 8, 2, [(9, 65), (16, 129), (13, 100), (16, 64), (12, 7000)], (16, BIG)),
    ("list", 8, 2, [(300, 301), (1, 100), (33, 65)], (300, BIG)),
    ("list", 8, 2, [(321, 321), (65, 129), (97, 127)], (321, BIG)),
    ("list", 3, 1, [(400, 5001), (1, 2050), (129, 2047)], (400, BIG)),                # keys in ranges
    ("steps 1 + list", 8, 2, SEQS + [(300, 301)] + [(1, 30 + i) for i in range(20)], (300, BIG)),
]


def ids(c):
    return "%s %d %d" % (c[0], c[1], c[3][0][0])


def width(seqs):
    return max(-(-t // 16) for _, t in seqs) + BIG // 16


@pytest.mark.parametrize("case", PATHS, ids=ids)
def test_paths_are_the_ones_named(case):
    name, hq, hkv, seqs, hints = case
    assert choice.path(hq, hkv, seqs, hints, 16, width(seqs)) == name


def made(case, back, values):
    """A value in a dim of its own, of one KV head, at every sequence's key `back` from its end."""
    _, hq, hkv, seqs, _ = case
    b = ref.Batch(91 + back, hq, hkv, 16, seqs, table_extra=BIG // 16)
    for i, (_, t) in enumerate(seqs):
        for d, value in enumerate(values):
            if back < t:
                b.values[i][t - 1 - back, (i + d) % hkv, 7 * d + i % 7] = value
        b.put(i)
    return b


def check(b, hints, causal, what, out_dtype=torch.bfloat16, flags=0):
    kc, vc, bt, cu, lk = b.to(DEV)
    out, lse = pec.pec_attn_paged(b.q.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk, *hints, causal=causal, out_dtype=out_dtype, flags=flags)
    want = ref.attention(b, causal)
    got = out.cpu().double()
    assert bool((got.isnan() == want[0].isnan()).all()), "%s: NaN in other places" % what
    inf = want[0].isinf()
    assert bool((got[inf] == want[0][inf]).all()), "%s: an infinity of the other sign" % what
    ref.assert_attention(out, lse, want, what, plain=flags != 0)


@pytest.mark.gpu
@pytest.mark.parametrize("case", PATHS, ids=ids)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("back", [0, 1, 40])
def test_values_that_rows_see(case, causal, back):
    b = made(case, back, [INF, -INF, NAN])
    check(b, case[4], causal, "%s back %d" % (case[0], back))
    check(b, case[4], causal, "%s back %d fp32" % (case[0], back), torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
def test_the_plain_kernel(causal):
    for back in (0, 1):
        check(made(PATHS[4], back, [INF, -INF, NAN]), (0, 0), causal, "plain", flags=pec.PEC_FLAG_SIMPLE_KERNEL)


@pytest.mark.gpu
@pytest.mark.parametrize("case", PATHS, ids=ids)
def test_infinities_of_both_signs_in_a_sum_are_nan(case):
    b = made(case, 0, [INF])
    for i, (_, t) in enumerate(b.seqs):
        if t > 40:
            b.values[i][t - 40, i % b.hkv, i % 7] = -INF
        b.put(i)
    for causal in (True, False):
        check(b, case[4], causal, case[0])
