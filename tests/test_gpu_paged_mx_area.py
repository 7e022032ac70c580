"""The way through the workspace of a call on a cache in 4 bits (keys turned into bf16 there, then the list), with and without decode steps
launched apart: hidden and infinite values, offsets that fall, a workspace that other calls have used, two streams, replayed graphs."""
import functools
import math

import pytest
import torch

from mx_calls import way
from paged_mx_reference import MxBatch
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"
HINTS, ROOM, PAGE = (512, 30512), 100000, 64      # of calls that the estimates send there
ALONE = [(500, 500), (90, 333), (300, 310)]
BESIDE = [(1, 90), (500, 700), (1, 7), (2, 300), (1, 64), (300, 300), (0, 40), (1, 128), (1, 1)]


@functools.lru_cache(maxsize=2)
def width(seqs):
    return max(-(-t // PAGE) for _, t in seqs) + 500


def made(seed, seqs, hq=32, hkv=8):
    b = MxBatch(seed, hq, hkv, PAGE, list(seqs), spare_rows=2, table_extra=500)
    want = "steps, list" if len(seqs) > 4 else "list"
    assert way(hq, hkv, seqs, HINTS, PAGE, b.table.shape[1], ROOM, 2) == want
    return b


def workspace(b, fill=0xff):
    return torch.full((pec.pec_paged_mx_workspace_bytes(b.hq, b.hkv, len(b.seqs), b.total, ROOM),), fill, dtype=torch.uint8, device=DEV)


def run(b, causal=True, ws=None, held=None, out_dtype=torch.float32, **kw):
    cache, table, cu, len_k = held or b.to(DEV)
    ws = workspace(b) if ws is None else ws
    out = torch.full((b.total, b.hq, 128), 55.0, dtype=out_dtype, device=DEV)
    lse = torch.full((b.hq, b.total), 55.0, device=DEV)
    pec.pec_attn_paged_mx(b.q.to(DEV), pec.PagedCacheMx(*cache), table, cu, len_k, *HINTS, causal=causal, out_dtype=out_dtype, out=out, lse=lse,
                          workspace=ws, **kw)
    return out, lse


@pytest.mark.parametrize("seqs", [ALONE, BESIDE], ids=["alone", "beside"])
def test_values_that_some_rows_do_not_see(seqs):
    """NaN and infinite values among the new tokens: rows ahead of them have nothing of it, the others what they see."""
    b = made(61, seqs)
    for i, (n, t) in enumerate(b.seqs):
        if n < 5:
            continue
        pages, slots = b.where(i)
        for at, byte, group in ((t - 1, 255, 0), (t - n // 2 - 1, 255, 2), (t - n + 1, 254, 1), (t - 2, 253, 3)):
            b.v_scale[pages[at], :, group, slots[at]] = byte
            b.v[pages[at], slots[at], :, 16 * group:16 * group + 16] = 0x77      # 6 x 2^126 and more: infinite
            b.values[i][at, :, 32 * group:32 * group + 32] = math.nan if byte == 255 else math.inf
    want = attention(b)
    for dtype in (torch.float32, torch.bfloat16):
        out, lse = run(b, out_dtype=dtype)
        assert_attention(out, lse, want)
        got, inf = out[:b.rows].cpu().double(), want[0].isinf()
        assert bool((got[inf] == want[0][inf]).all()) and torch.equal(got.isnan(), want[0].isnan())
        assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


@pytest.mark.parametrize("seqs", [ALONE, BESIDE], ids=["alone", "beside"])
def test_keys_of_nan_make_rows_nan_that_see_them(seqs):
    b = made(62, seqs)
    clean = attention(b)
    i, (n, t) = 1, b.seqs[1]
    pages, slots = b.where(i)
    at, row = t - n + 40, int(b.cu[i]) + 40
    b.k_scale[pages[at], 5, 2, slots[at]] = 255
    out, lse = run(b)
    nan = torch.zeros(b.hq, b.total, dtype=torch.bool)
    nan[20:24, row:int(b.cu[i + 1])] = True
    assert torch.equal(lse.isnan().cpu(), nan) and torch.equal(out.isnan().any(-1).cpu(), nan.T) and torch.equal(out.isnan().all(-1).cpu(), nan.T)
    out, lse = out.cpu(), lse.cpu()
    rows = slice(0, b.rows)
    out[rows][nan.T[rows]], lse[:, rows][nan[:, rows]] = clean[0][nan.T[rows]].float(), clean[1][nan[:, rows]].float()
    assert_attention(out, lse, clean, "rows that do not see it")


@pytest.mark.parametrize("seqs", [[(90, 0), (500, 500), (300, 310)], [(500, 500), (300, 310), (90, 0)]], ids=["first", "last"])
def test_a_sequence_without_keys(seqs):
    """New tokens and no key: the rows are empty, also where the area is full to its last page."""
    b = made(63, seqs)
    exact = 64 * (13 - len(seqs))      # 13 pages are what the two sequences with keys take
    assert way(32, 8, seqs, HINTS, PAGE, b.table.shape[1], exact, 2) == "list"
    sizes = [pec.pec_paged_mx_workspace_bytes(32, 8, len(seqs), b.total, room) for room in (0, exact, ROOM)]
    assert 13 * 2 * 8 * PAGE * 256 <= sizes[1] - sizes[0] < 14 * 2 * 8 * PAGE * 256
    for size in sizes[1:]:
        for causal in (True, False):
            out, lse = run(b, causal, torch.full((size,), 0xff, dtype=torch.uint8, device=DEV))
            assert_attention(out, lse, attention(b, causal), "%d bytes" % size)
            assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())


def test_more_sequences_than_the_area_kernel_has_lanes():
    seqs = [(9 + i % 3, (13 * i) % 90 + (0 if i % 50 == 7 else 9)) for i in range(1100)]
    b = MxBatch(64, 8, 2, 16, seqs, spare_rows=1, table_extra=1950)
    room, hints = 700000, (2000, 30512)
    cache, table, cu, len_k = b.to(DEV)
    want = attention(b)
    for total_k in (room, 10000):      # for all; for the first of them
        assert way(8, 2, seqs, hints, 16, b.table.shape[1], total_k, 1) == "steps, list"
        ws = torch.full((pec.pec_paged_mx_workspace_bytes(8, 2, len(seqs), b.total, total_k),), 0xff, dtype=torch.uint8, device=DEV)
        out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), pec.PagedCacheMx(*cache), table, cu, len_k, *hints, out_dtype=torch.float32, workspace=ws)
        assert_attention(out, lse, want)


def test_offsets_that_fall_stay_in_bounds():
    """Malformed offsets and lengths: nothing behind the packed rows, outside the results or outside the workspace is touched."""
    for seqs in (ALONE, BESIDE):
        b = made(65, seqs)
        cache, table, _, _ = b.to(DEV)
        held, q, n = pec.PagedCacheMx(*cache), b.q.to(DEV), len(seqs)
        size = pec.pec_paged_mx_workspace_bytes(b.hq, b.hkv, n, b.total, ROOM)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        fall = [0, 700, 3, 600, 10, 800, 0, 802, 9, 802][:n] + [802]
        wild = [-5, 2 ** 30, -7, 0, 2 ** 31 - 1, 1, 2 ** 31 - 1, -2 ** 31, 700, 3][:n + 1]
        for cu, len_k in ((fall, [700, 300, 33, 5, 20, 500, 600, 1, 64][:n]), (wild, [-4, 2 ** 31 - 1, 0, 10 ** 6, 64, -1, 900, 2 ** 31 - 1, 5][:n])):
            ws = torch.full((size + 4096,), 9, dtype=torch.uint8, device=DEV)
            guard = torch.full((b.total + 8, b.hq, 128), 9.0, dtype=torch.bfloat16, device=DEV)
            lguard = torch.full((b.hq * b.total + 64,), 9.0, device=DEV)
            pec.pec_attn_paged_mx(q, held, table, i32(cu), i32(len_k), *HINTS, out=guard[:b.total], lse=lguard[:b.hq * b.total].view(b.hq, b.total),
                                  workspace=ws[:size])
            torch.cuda.synchronize()
            assert bool((guard[b.total:] == 9).all()) and bool((lguard[b.hq * b.total:] == 9).all()) and bool((ws[size:] == 9).all())


def test_a_workspace_that_other_calls_have_used():
    """The same call again, after calls whose sequences had other pages of the area: equal to the last bit."""
    b, other = made(66, BESIDE), made(67, BESIDE[::-1])
    ws, held = workspace(b), b.to(DEV)
    first = run(b, ws=ws, held=held)
    assert_attention(*first, attention(b))
    for causal in (True, False):
        run(other, causal, ws=ws)
        again = run(b, ws=ws, held=held)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_two_streams_at_once():
    b = made(68, BESIDE)
    held, streams = b.to(DEV), [torch.cuda.Stream() for _ in range(2)]
    spaces = [workspace(b), workspace(b)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(run(b, ws=spaces[i % 2], held=held))
    torch.cuda.synchronize()
    want = attention(b)
    for out, lse in got:
        assert_attention(out, lse, want)
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])


@pytest.mark.parametrize("seqs", [ALONE, BESIDE], ids=["alone", "beside"])
def test_replayed_with_other_lengths(seqs):
    """A captured call replayed while lengths, offsets and queries change on the device, with eager calls between: every replay equals the
    eager call to the last bit and meets the definition."""
    b = made(69, seqs)
    (cache, table, cu, len_k), q, ws = b.to(DEV), b.q.to(DEV), workspace(b)
    held = pec.PagedCacheMx(*cache)
    out, lse = torch.empty(b.total, b.hq, 128, device=DEV), torch.empty(b.hq, b.total, device=DEV)
    call = lambda o, l, w: pec.pec_attn_paged_mx(q, held, table, cu, len_k, *HINTS, out_dtype=torch.float32, out=o, lse=l, workspace=w)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, lse, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    g = torch.Generator().manual_seed(1)
    for step in range(4):
        b.seqs = [(n - min(n, 3 * step * (i % 2)), t - min(t, 11 * step * ((i + 1) % 3))) for i, (n, t) in enumerate(seqs)]
        ends = torch.cumsum(torch.tensor([0] + [n for n, _ in b.seqs]), 0).to(torch.int32)
        b.cu, b.rows = ends, int(ends[-1])
        b.q = torch.randn(b.total, b.hq, 128, generator=g).to(torch.bfloat16)
        cu.copy_(ends)
        len_k.copy_(torch.tensor([t for _, t in b.seqs], dtype=torch.int32))
        q.copy_(b.q)
        graph.replay()
        eager_out, eager_lse = torch.empty_like(out), torch.empty_like(lse)
        call(eager_out, eager_lse, workspace(b))
        torch.cuda.synchronize()
        assert torch.equal(out[:b.rows], eager_out[:b.rows]) and torch.equal(lse[:, :b.rows], eager_lse[:, :b.rows])
        short = MxBatch.__new__(MxBatch)
        short.hq, short.hkv, short.rows, short.seqs, short.cu, short.q = b.hq, b.hkv, b.rows, b.seqs, b.cu, b.q
        short.keys, short.values = [k[:t] for k, (_, t) in zip(b.keys, b.seqs)], [v[:t] for v, (_, t) in zip(b.values, b.seqs)]
        assert_attention(out, lse, attention(short), "step %d" % step)
