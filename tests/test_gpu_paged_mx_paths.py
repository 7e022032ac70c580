"""Every way in which attention over a cache in 4 bits is cut, and what can go wrong in each."""
import math

import pytest
import torch

import mx_choice
from paged_mx_reference import MxBatch, quantise, values
from paged_reference import assert_attention, attention
from paper_2409_15104_amd import binding as pec

pytestmark = pytest.mark.gpu
DEV = "cuda"


def run(b, hints=(0, 0), causal=True, by_head=False, room=0, out_dtype=torch.float32, **kw):
    held, table, cu, len_k = b.to(DEV, by_head)
    cache = pec.PagedCacheMx(*held)
    ws = torch.full((pec.pec_paged_mx_workspace_bytes(b.hq, b.hkv, len(b.seqs), b.total, room),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((b.total, b.hq, 128), 55.0, dtype=out_dtype, device=DEV)
    lse = torch.full((b.hq, b.total), 55.0, device=DEV)
    pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, max_len_q=hints[0], max_len_k=hints[1], causal=causal, out_dtype=out_dtype,
                          out=out, lse=lse, workspace=ws, **kw)
    assert bool((out[b.rows:] == 55).all()) and bool((lse[:, b.rows:] == 55).all())
    return out, lse


CASES = [      # heads, KV heads, page, by head, sequences, hints, room, path
    (32, 8, 16, False, [(1, 90), (1, 33), (1, 128)], (1, 128), 0, "units 1 8"),
    (32, 8, 16, True, [(1, 40 + 7 * i % 50) for i in range(40)], (1, 90), 0, "units 1 4"),
    (32, 8, 16, False, [(1, 40 + 7 * i % 50) for i in range(40)], (1, 90), 0, "units 1 4"),
    (8, 8, 32, False, [(20, 90), (31, 31), (5, 300)], (31, 300), 0, "units 2 4"),
    (16, 2, 16, True, [(40, 95), (6, 6), (17, 230)], (40, 230), 0, "units 3 4"),
    (8, 8, 8, False, [(1, 300), (1, 7), (1, 64)], (1, 300), 0, "spans 1"),
    (6, 2, 8, False, [(30, 300), (7, 7), (1, 64)], (30, 300), 0, "spans 3"),
    (4, 2, 8, True, [(10, 300), (7, 7), (1, 64)], (10, 300), 0, "spans 2"),
    (16, 8, 16, False, [(1, 5000), (1, 90), (1, 2222), (1, 16)], (1, 5000), 0, "spans 1"),
    (8, 1, 64, True, [(2, 9000), (1, 40), (2, 700)], (2, 9000), 0, "spans 1"),
    (5, 1, 16, False, [(5, 9000), (2, 40), (5, 700)], (5, 9000), 0, "spans 2"),
    (8, 1, 32, False, [(6, 9000), (6, 100), (1, 3000)], (6, 9000), 0, "spans 3"),
    (8, 2, 32, True, [(100, 9000)], (100, 9000), 0, "spans 3"),
    (32, 8, 64, False, [(512, 700)], (512, 30512), 700, "list"),
    (32, 8, 64, True, [(512, 700)], (512, 30512), 40000, "list"),        # room for all that the table could hold
    (32, 8, 64, False, [(512, 700)], (512, 30512), 300, "list"),         # no room: the steps take it
    (8, 2, 16, False, [(1, 300)] * 4 + [(150, 150), (90, 700)], (150, 9000), 0, "beside"),
    (8, 2, 16, True, [(1, 300)] * 6 + [(150, 20000)], (150, 20000), 0, "beside"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_%d_%d" % (c[7].replace(" ", "_"), c[0], c[2]))
def test_path(case):
    hq, hkv, page, by_head, seqs, hints, room, path = case
    b = MxBatch(21, hq, hkv, page, seqs, spare_rows=2, table_extra=2 if path != "list" else 580)
    assert mx_choice.path(hq, hkv, seqs, hints, page, b.table.shape[1], 2, room > 0) == path
    out, lse = run(b, hints, by_head=by_head, room=room)
    assert_attention(out, lse, attention(b), path)
    out, lse = run(b, hints, causal=False, by_head=by_head, room=room, out_dtype=torch.bfloat16)
    assert_attention(out, lse, attention(b, causal=False), path)


@pytest.mark.parametrize("hints", [(1, 16), (3, 64), (200, 10 ** 6)])
def test_hints_that_are_wrong_change_nothing(hints):
    b = MxBatch(22, 8, 2, 16, [(1, 500), (70, 170), (3, 3), (90, 400), (1, 1)])
    for room in (0, 2000):
        assert_attention(*run(b, hints, room=room), attention(b), str(hints))


@pytest.mark.parametrize("room", [0, 3000])
@pytest.mark.parametrize("hq,hkv,page", [(8, 2, 16), (8, 8, 8), (24, 1, 32)])
def test_hidden_values_reach_no_row(hq, hkv, page, room):
    """New tokens whose values are NaN or too large for bf16: rows ahead of them have nothing of it, the others what they see."""
    b = MxBatch(23, hq, hkv, page, [(40, 140), (5, 33), (70, 70), (3, 900)])
    for i, (n, t) in enumerate(b.seqs):
        pages, slots = b.where(i)
        for at, byte, group in ((t - 1, 255, 0), (t - n // 2 - 1, 255, 2), (t - n + 1, 254, 1), (t - 2, 253, 3)):
            b.v_scale[pages[at], :, group, slots[at]] = byte
            b.v[pages[at], slots[at], :, 16 * group:16 * group + 16] = 0x77      # 6 x 2^126 and more: infinite
            b.values[i][at, :, 32 * group:32 * group + 32] = math.nan if byte == 255 else math.inf
    out, lse = run(b, (70, 900), room=room)
    assert_attention(out, lse, attention(b), "hidden")
    out, lse = run(b, (70, 900), room=room, flags=pec.PEC_FLAG_SIMPLE_KERNEL)
    assert_attention(out, lse, attention(b), "hidden", plain=True)


def test_keys_of_nan_make_rows_nan_that_see_them():
    b = MxBatch(24, 8, 2, 16, [(4, 100), (1, 40)])
    pages, slots = b.where(0)
    b.k_scale[pages[98], 1, 2, slots[98]] = 255      # the new token before the last one, second KV head
    out, lse = run(b, (4, 100))
    nan = torch.isnan(lse.cpu())
    want = torch.zeros_like(nan)
    want[4:, 2:4] = True
    assert torch.equal(nan, want)
    assert torch.equal(torch.isnan(out.cpu()).all(-1), want.T) and torch.equal(torch.isnan(out.cpu()).any(-1), want.T)


def test_more_sequences_than_a_wavefront_holds():
    seqs = [(i % 3, (37 * i) % 200 + 3) for i in range(150)] + [(2, 3000)]
    b = MxBatch(25, 4, 2, 16, seqs, spare_rows=1)
    for hints in ((2, 3000), (2, 300)):
        assert_attention(*run(b, hints), attention(b), str(hints))


def test_scale_and_strided_queries():
    b = MxBatch(26, 8, 4, 16, [(3, 77), (1, 200)])
    held, table, cu, len_k = b.to(DEV)
    wide = torch.randn(b.total, 16, 128).to(torch.bfloat16).to(DEV)
    wide[:, :8] = b.q.to(DEV)
    out, lse = pec.pec_attn_paged_mx(wide[:, :8], pec.PagedCacheMx(*held), table, cu, len_k, scale=0.03)
    assert_attention(out, lse, attention(b, scale=0.03))


def test_a_pool_beyond_32_bits():
    """Pages 6 GB apart: offsets of codes and scales need 64 bits."""
    page, hkv = 16, 2
    codes = torch.zeros((3 << 30) + 4096, dtype=torch.uint8, device=DEV)
    stride = 3 << 29
    k = codes.as_strided((3, page, hkv, 64), (stride, hkv * 64, 64, 1))
    v = codes[2048:].as_strided((3, page, hkv, 64), (stride, hkv * 64, 64, 1))
    scales = torch.zeros((5 << 30) + 4096, dtype=torch.uint8, device=DEV)
    ss = 5 << 29
    ks = scales.as_strided((3, hkv, 4, page), (ss, 4 * page, page, 1))
    vs = scales[1024:].as_strided((3, hkv, 4, page), (ss, 4 * page, page, 1))
    cache = pec.PagedCacheMx(k, v, ks, vs)
    b = MxBatch(27, 4, hkv, page, [(40, 40)], spare_pages=0, wild=False)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    cu, len_k = b.cu.to(DEV), b.len_k.to(DEV)
    x, y = b.raw[0]
    pec.pec_paged_append_mx(x.to(DEV), y.to(DEV), cache, table, cu, len_k)
    kk, vv = pec.pec_paged_read_mx(cache, table, cu, len_k, total_q=40)
    assert torch.equal(kk.cpu().double(), b.keys[0]) and torch.equal(vv.cpu().double(), b.values[0])
    out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k)
    assert_attention(out, lse, attention(b))
    out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, cu, len_k, flags=pec.PEC_FLAG_SIMPLE_KERNEL)
    assert_attention(out, lse, attention(b), plain=True)


def layer_steps(cache, table, state, q, k, v, ws, out, lse, rope):
    """One step of a layer: append, attention, and the new tokens read back."""
    cu, len_k = state
    pec.pec_paged_append_mx(k, v, cache, table, cu, len_k, norm_rope=rope, q=q, q_out=q)
    pec.pec_attn_paged_mx(q, cache, table, cu, len_k, max_len_q=1, max_len_k=200, out_dtype=out.dtype, out=out, lse=lse,
                          workspace=ws)
    return pec.pec_paged_read_mx(cache, table, cu, len_k, total_q=q.shape[0])


def test_a_run_of_steps_captured_and_replayed():
    """A prompt, then decode steps from a graph whose lengths move on the device; every replay against the definition, with eager work
    on the same cache between the replays."""
    hq, hkv, page, n_steps = 8, 2, 16, 5
    seqs = [(1, 50 + n_steps), (1, 17 + n_steps), (1, 3 + n_steps)]
    b = MxBatch(28, hq, hkv, page, seqs)
    fill = lambda *s: torch.full(s, 255, dtype=torch.uint8, device=DEV)  # noqa: E731
    cache = pec.PagedCacheMx(fill(b.n_pages, page, hkv, 64), fill(b.n_pages, page, hkv, 64), fill(b.n_pages, hkv, 4, page), fill(b.n_pages, hkv, 4, page))
    table = b.table.to(DEV)
    # the prompts, in one call
    prompt = [t - n_steps for _, t in seqs]
    cu0 = torch.tensor([0] + torch.cumsum(torch.tensor(prompt), 0).tolist(), dtype=torch.int32, device=DEV)
    len0 = torch.tensor(prompt, dtype=torch.int32, device=DEV)
    cat = lambda i, lo, hi: torch.cat([b.raw[s][i][lo(s):hi(s)] for s in range(3)]).to(DEV)  # noqa: E731
    pec.pec_paged_append_mx(cat(0, lambda s: 0, lambda s: prompt[s]), cat(1, lambda s: 0, lambda s: prompt[s]), cache, table, cu0, len0)
    cu = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV)
    len_k = len0.clone()
    g = torch.Generator().manual_seed(4)
    q_all = torch.randn(n_steps, 3, hq, 128, generator=g).to(torch.bfloat16).to(DEV)
    step_k = [cat(0, lambda s: prompt[s] + i, lambda s: prompt[s] + i + 1) for i in range(n_steps)]
    step_v = [cat(1, lambda s: prompt[s] + i, lambda s: prompt[s] + i + 1) for i in range(n_steps)]
    q, k, v = torch.empty_like(q_all[0]), torch.empty_like(step_k[0]), torch.empty_like(step_v[0])
    ws = torch.empty(pec.pec_paged_mx_workspace_bytes(hq, hkv, 3, 3), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(3, hq, 128, dtype=torch.float32, device=DEV), torch.empty(hq, 3, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    spare = cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone()
    with torch.cuda.stream(side):      # once outside the graph, on the prompts' last tokens again
        layer_steps(cache, table, (cu, len_k), q.zero_(), k.zero_(), v.zero_(), ws, out, lse, None)
    torch.cuda.current_stream().wait_stream(side)
    for held, was in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), spare):
        held.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        back = layer_steps(cache, table, (cu, len_k), q, k, v, ws, out, lse, None)
    for i in range(n_steps):
        q.copy_(q_all[i])
        k.copy_(step_k[i])
        v.copy_(step_v[i])
        len_k += 1
        graph.replay()
        eager, _ = pec.pec_attn_paged_mx(q, cache, table, cu, len_k, max_len_q=1, max_len_k=200, out_dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(eager, out)
        now = MxBatch.__new__(MxBatch)
        now.hq, now.hkv, now.rows, now.seqs = hq, hkv, 3, [(1, prompt[s] + i + 1) for s in range(3)]
        now.cu, now.q = cu.cpu(), q.cpu()
        now.keys = [b.keys[s][:prompt[s] + i + 1] for s in range(3)]
        now.values = [b.values[s][:prompt[s] + i + 1] for s in range(3)]
        assert_attention(out, lse, attention(now), "step %d" % i)
        for got, held in zip(back, (b.keys, b.values)):
            assert torch.equal(got.cpu().double(), torch.stack([held[s][prompt[s] + i] for s in range(3)]))


def test_two_streams_at_once():
    """Two calls on their own streams with a workspace each, on one cache."""
    b = MxBatch(29, 16, 4, 16, [(1, 700), (60, 900), (1, 3)])
    held, table, cu, len_k = b.to(DEV)
    cache, q = pec.PagedCacheMx(*held), b.q.to(DEV)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        got.append(pec.pec_attn_paged_mx(q, cache, table, cu, len_k, total_k=2000 * (i % 2), out_dtype=torch.float32, stream=streams[i % 2]))
    torch.cuda.synchronize()
    ref = attention(b)
    for out, lse in got:
        assert_attention(out, lse, ref)


def test_rounding_on_the_way_in_is_what_attention_reads():
    """append, then attention, against the definition on rounded rows: one sequence's prompt in two chunks."""
    b = MxBatch(30, 8, 2, 16, [(45, 100)])
    z = lambda *s: torch.full(s, 255, dtype=torch.uint8, device=DEV)  # noqa: E731
    cache = pec.PagedCacheMx(z(b.n_pages, 16, 2, 64), z(b.n_pages, 16, 2, 64), z(b.n_pages, 2, 4, 16), z(b.n_pages, 2, 4, 16))
    k, v = [t.to(DEV) for t in b.raw[0]]
    table = b.table.to(DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    pec.pec_paged_append_mx(k[:55], v[:55], cache, table, i32(0, 55), i32(55))
    pec.pec_paged_append_mx(k[55:], v[55:], cache, table, i32(0, 45), i32(100))
    out, lse = pec.pec_attn_paged_mx(b.q.to(DEV), cache, table, i32(0, 45), i32(100))
    assert_attention(out, lse, attention(b))
    c, s = quantise(b.raw[0][0])
    assert torch.equal(values(c, s), b.keys[0])


@pytest.mark.parametrize("flags", [0, pec.PEC_FLAG_SIMPLE_KERNEL])
@pytest.mark.parametrize("page", [8, 16])
def test_tables_without_a_page(page, flags):
    """No page for any token: nothing is stored, rows come back as zeros, every row is empty."""
    z = lambda *s: torch.full(s, 255, dtype=torch.uint8, device=DEV)  # noqa: E731
    cache = pec.PagedCacheMx(z(2, page, 2, 64), z(2, page, 2, 64), z(2, 2, 4, page), z(2, 2, 4, page))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    table, cu, len_k = torch.empty(2, 0, dtype=torch.int32, device=DEV), i32(0, 3, 5), i32(0, 90)
    q, k = torch.ones(6, 4, 128, dtype=torch.bfloat16, device=DEV), torch.ones(6, 2, 128, dtype=torch.bfloat16, device=DEV)
    pec.pec_paged_append_mx(k, k, cache, table, cu, len_k)
    assert bool((cache.k == 255).all()) and bool((cache.v_scale == 255).all())
    back = pec.pec_paged_read_mx(cache, table, cu, len_k, k=k.clone(), v=k.clone())
    for t in back:
        assert bool((t[:5] == 0).all()) and bool((t[5:] == 1).all())
    for causal in (True, False):
        out, lse = torch.ones_like(q), torch.ones(4, 6, device=DEV)
        pec.pec_attn_paged_mx(q, cache, table, cu, len_k, causal=causal, flags=flags, out=out, lse=lse)
        assert bool((out[:5] == 0).all()) and bool((lse[:, :5] == -math.inf).all())
        assert bool((out[5:] == 1).all()) and bool((lse[:, 5:] == 1).all())


def test_offsets_that_fall_stay_in_bounds():
    """Malformed offsets and lengths: whatever comes out, nothing behind the last packed row or outside the results is touched."""
    b = MxBatch(31, 8, 2, 16, [(1, 90), (40, 70), (3, 33), (1, 5), (20, 20)], spare_rows=3)
    held, table, _, _ = b.to(DEV)
    cache, q = pec.PagedCacheMx(*held), b.q.to(DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for cu, len_k in ((i32(0, 50, 3, 60, 10, 68), i32(90, 70, 33, 5, 20)), (i32(-5, 2 ** 30, -7, 0, 2 ** 31 - 1, 1), i32(-4, 2 ** 31 - 1, 0, 10 ** 6, 64))):
        for room in (0, 500):
            guard = torch.full((b.total + 8, 8, 128), 9.0, dtype=torch.bfloat16, device=DEV)
            lguard = torch.full((8 * b.total + 64,), 9.0, device=DEV)
            out, lse = guard[:b.total], lguard[:8 * b.total].view(8, b.total)
            pec.pec_attn_paged_mx(q, cache, table, cu, len_k, out=out, lse=lse, total_k=room)
            torch.cuda.synchronize()
            assert bool((guard[b.total:] == 9).all()) and bool((lguard[8 * b.total:] == 9).all())


def test_results_do_not_depend_on_what_ran_before():
    """The same call twice, with other calls on the same workspace between: equal to the last bit."""
    b = MxBatch(32, 16, 8, 16, [(1, 6000), (1, 40), (6, 900), (6, 6)])
    held, table, cu, len_k = b.to(DEV)
    cache, q = pec.PagedCacheMx(*held), b.q.to(DEV)
    ws = torch.empty(pec.pec_paged_mx_workspace_bytes(16, 8, 4, b.total, 3000), dtype=torch.uint8, device=DEV)
    call = lambda **kw: pec.pec_attn_paged_mx(q, cache, table, cu, len_k, out_dtype=torch.float32, workspace=ws, **kw)  # noqa: E731
    first = call(max_len_q=6, max_len_k=6000)
    for other in (dict(max_len_q=1, max_len_k=40), dict(), dict(max_len_q=14, max_len_k=9000)):
        call(**other)
        again = call(max_len_q=6, max_len_k=6000)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
