"""Calls on a cache in 4 bits that are taken apart: steps by themselves, and beside them chunks in every way they are worked on."""
import functools

import pytest
import torch

from mx_calls import way
from paged_mx_reference import MxBatch
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEPS = [(1, 90), (1, 700), (3, 300), (1, 64), (0, 50), (2, 2)]
CHUNKS = [(300, 6000), (280, 5000), (250, 7000)]
SEQS = STEPS[:3] + CHUNKS[:1] + STEPS[3:] + CHUNKS[1:] + STEPS
SMALL = STEPS[:3] + [(70, 170)] + STEPS[3:] + [(150, 150), (33, 400)] + STEPS


@functools.lru_cache(maxsize=4)
def made(hq, hkv, page, seqs, table_extra):
    b = MxBatch(51, hq, hkv, page, list(seqs), spare_rows=2, table_extra=table_extra)
    return b, {causal: attention(b, causal) for causal in (True, False)}


def check(b, ref, hints, room, causal=True, by_head=False, dtype=torch.float32):
    held, table, cu, len_k = b.to(DEV, by_head)
    ws = torch.full((pec.pec_paged_mx_workspace_bytes(b.hq, b.hkv, len(b.seqs), b.total, room),), 0xff, dtype=torch.uint8, device=DEV)
    out, lse = torch.full((b.total, b.hq, 128), 55.0, dtype=dtype, device=DEV), torch.full((b.hq, b.total), 55.0, device=DEV)
    pec.pec_attn_paged_mx(b.q.to(DEV), pec.PagedCacheMx(*held), table, cu, len_k, *hints, causal=causal, out_dtype=dtype, out=out, lse=lse,
                          workspace=ws)
    assert_attention(out, lse, ref[causal], "room %d" % room)
    assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("room,by_head", [(12500, False), (20000, True), (100000, False)])
def test_chunks_with_room_for_some_beside_steps(room, by_head, causal):
    """Of three chunks two find room, all, all with the widest table."""
    b, ref = made(16, 8, 64, tuple(SEQS), 300)
    hints = (b.total, 25000)
    assert way(16, 8, b.seqs, hints, 64, b.table.shape[1], room, 2) == "steps, list"
    check(b, ref, hints, room, causal, by_head)


def test_room_for_every_chunk_for_certain():
    """As much as the widest sequences would need that the table has room for: nothing is launched for those without room."""
    b, ref = made(16, 8, 64, tuple(SEQS), 300)
    hints, room = (b.total, 25000), 64 * (b.total // 9 + 1) * b.table.shape[1]
    assert way(16, 8, b.seqs, hints, 64, b.table.shape[1], room, 2) == "steps, list"
    check(b, ref, hints, room, dtype=torch.bfloat16)


CASES = [      # heads, KV heads, page, hints, room, way
    (16, 2, 16, (None, 0), 0, "steps, spans 3"),
    (16, 8, 16, (150, 0), 700, "steps, units 3"),
    (16, 2, 8, (150, 8000), 0, "steps, spans 3"),
    (12, 4, 16, (150, 8000), 0, "steps, units 3"),
    (32, 8, 16, (150, 0), 700, "steps, units 3"),
    (8, 8, 16, (150, 8000), 0, "spans 3"),
    (16, 2, 16, (150, 700), 0, "units 3"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_%d_%d_%d" % (c[5].replace(", ", "_").replace(" ", "_"), c[0], c[2], c[4]))
def test_ways(case):
    hq, hkv, page, hints, room, want = case
    b, ref = made(hq, hkv, page, tuple(SMALL), 20000 // page)
    hints = (b.total if hints[0] is None else hints[0], hints[1])
    assert way(hq, hkv, b.seqs, hints, page, b.table.shape[1], room, 2) == want
    for causal in (True, False):
        check(b, ref, hints, room, causal)


def test_decode_steps_without_hints():
    seqs = [(1, 1 + 37 * i % 800) for i in range(70)]
    b = MxBatch(52, 8, 2, 16, seqs, spare_rows=0, table_extra=600)
    assert way(8, 2, seqs, (0, 0), 16, b.table.shape[1]) == "steps, units 3"
    check(b, {True: attention(b)}, (0, 0), 0)
