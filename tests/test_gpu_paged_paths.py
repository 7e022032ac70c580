"""Every way in which pec_attn_paged cuts its work (units of 32 rows with eight and four wavefronts, spans of 32 and 64 rows, the work
list, whole and in ranges, and both together), on batches that reach their corners, and calls as a server makes them: captured and
replayed, on several streams, one behind the other through one workspace."""
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


def attend(b, hints, causal=True, out_dtype=torch.bfloat16, by_head=False, **kw):
    kc, vc, bt, cu, lk = b.to(DEV, by_head)
    out = torch.full(b.q.shape, 5.0, dtype=out_dtype, device=DEV)
    lse = torch.full((b.hq, b.total), 5.0, device=DEV)
    pec.pec_attn_paged(b.q.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk, *hints, causal=causal, out_dtype=out_dtype, out=out, lse=lse, **kw)
    assert bool((out[b.rows:] == 5).all()) and bool((lse[:, b.rows:] == 5).all())
    return out, lse


BIG = 8000      # keys that every block table here has room for, more than calls in units take
# path, hq, hkv, page, sequences (new, all), hints: the hints choose the path
PATHS = [
    ("units 8", 8, 2, 16, [(1, 700), (9, 40), (70, 300)], (70, 700)),
    ("units 4", 40, 8, 16, [(150, 200), (60, 90), (1, 30)], (150, 200)),
    ("units 8", 4, 4, 8, [(1, 1 + i % 50) for i in range(60)], (1, 50)),
    ("units 4", 4, 1, 32, [(1, 1 + i % 70) for i in range(4300)], (300, 70)),       # more than 4,096 sequences
    ("steps 1", 8, 2, 16, [(1, 700), (2, 40), (1, 5000), (8, 8)], (8, BIG)),
    ("steps 1", 2, 1, 8, [(1, 1 + i % 90) for i in range(4300)], (1, BIG)),
    ("steps 1", 10, 2, 64, [(6, 700), (3, 2), (2, 0)], (6, BIG)),                    # rows without a key, a sequence without one
    ("steps 2", 10, 2, 16, [(12, 300), (7, 7), (13, 1000), (30, 400)], (12, BIG)),   # more row tiles than the hint says
    ("steps 2", 64, 1, 16, [(1, 3000), (1, 33)], (1, BIG)),
    ("list", 8, 2, 16, [(300, 400), (20, 900)], (300, BIG)),
    ("list", 128, 1, 32, [(1, 300), (9, 50)], (9, BIG)),                             # a group of 128
    ("list", 3, 1, 16, [(400, 5000), (1, 2000)], (400, BIG)),                     # keys cut into ranges, no rows but one in a tile
    ("steps 1 + list", 8, 2, 16, [(300, 300), (1, 900), (8, 40), (9, 40), (1, 1), (200, 6000)], (300, BIG)),
    ("steps 2 + list", 40, 1, 16, [(90, 300), (1, 900), (1, 40), (2, 40), (1, 1)], (90, BIG)),
    ("steps 1 + list", 4, 2, 16, [(600, 600)] + [(1, 1 + i) for i in range(1500)], (600, BIG)),     # more sequences than the builder holds at once
]


@pytest.mark.parametrize("case", PATHS, ids=lambda c: c[0])
@pytest.mark.parametrize("causal", [True, False])
def test_paths(case, causal):
    name, hq, hkv, page, seqs, hints = case
    b = ref.Batch(hq + len(seqs), hq, hkv, page, seqs, spare_rows=1, table_extra=BIG // page)
    want = ref.attention(b, causal)
    ref.assert_attention(*attend(b, hints, causal), want, name)
    ref.assert_attention(*attend(b, hints, causal, torch.float32, by_head=True), want, name + " fp32")


# the same paths, sequences of several tokens each
HIDDEN = [("units 8", [(6, 90), (40, 40), (70, 200)], (70, 200)), ("steps 1", [(6, 90), (9, 300), (16, 16)], (16, BIG)),
          ("steps 2", [(20, 90), (30, 70), (31, 300)], (32, BIG)), ("list", [(200, 310), (80, 80), (300, 5300)], (600, BIG))]


@pytest.mark.parametrize("case", HIDDEN, ids=lambda c: c[0])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_that_a_row_does_not_see(case, value):
    _, seqs, hints = case
    b = ref.Batch(31, 4, 2, 16, seqs, table_extra=BIG // 16)
    for i, (n, t) in enumerate(seqs):
        for back in (0, n // 2, n - 2):
            b.values[i][t - 1 - back, i % 2, 3 + back % 100] = value
        b.put(i)
    ref.assert_attention(*attend(b, hints), ref.attention(b), case[0])


@pytest.mark.parametrize("case", HIDDEN, ids=lambda c: c[0])
def test_nan_in_queries_and_keys_stays_in_its_rows(case):
    _, seqs, hints = case
    b = ref.Batch(32, 4, 2, 16, seqs, table_extra=BIG // 16)
    clean = ref.attention(b)
    b.q[2, 1, 7] = float("nan")
    n, t = seqs[1]
    b.keys[1][t - 3, 1] = float("nan")                # seen by the last three rows of KV head 1
    b.put(1)
    out, lse = attend(b, hints)
    bad = torch.zeros(b.rows, 4, dtype=torch.bool)
    bad[2, 1] = True
    bad[int(b.cu[2]) - 3:int(b.cu[2]), 2:] = True
    assert torch.equal(out.cpu().isnan().all(dim=-1), bad) and torch.equal(out.cpu().isnan().any(dim=-1), bad)
    assert torch.equal(lse.cpu().isnan(), bad.T)
    o, l = out.cpu().clone(), lse.cpu().clone()
    o[bad], l[bad.T] = clean[0][bad].to(o.dtype), clean[1][bad.T].float()
    ref.assert_attention(o, l, clean, case[0])


@pytest.mark.parametrize("case", HIDDEN, ids=lambda c: c[0])
def test_same_bits_whatever_the_workspace_held_and_whatever_ran_before(case):
    _, seqs, hints = case
    b = ref.Batch(33, 4, 2, 16, seqs, table_extra=BIG // 16)
    other = ref.Batch(34, 4, 2, 16, [(5, 400), (100, 100), (1, 3000)])
    n = max(pec.pec_paged_workspace_bytes(4, 2, len(x.seqs), x.total) for x in (b, other))
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    first = attend(b, hints, workspace=ws)
    attend(other, (0, 0), workspace=ws)
    ws.random_(0, 256)
    again = attend(b, hints, workspace=ws)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_streams_with_workspaces_of_their_own():
    jobs = [(ref.Batch(40 + i, 4, 2, 16, c[1], table_extra=BIG // 16), c[2]) for i, c in enumerate(HIDDEN)]
    alone = [attend(b, h) for b, h in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    held = []
    for b, _ in jobs:
        held.append((pec.PagedCache(*b.to(DEV)[:2]), b.to(DEV)[2:], b.q.to(DEV)))
    torch.cuda.synchronize()
    for _ in range(5):
        results = []
        for s, (b, h), (cache, meta, q) in zip(streams, jobs, held):
            with torch.cuda.stream(s):
                results.append(pec.pec_attn_paged(q, cache, *meta, *h))
        torch.cuda.synchronize()
        for (o, l), (o1, l1) in zip(results, alone):
            assert torch.equal(o, o1) and torch.equal(l, l1)


def angles(n):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    return torch.cat([a.cos(), a.sin()], dim=1).float()


class Layer:
    """A layer's attention step as a server runs it: norms, rotation and append, then attention, buffers kept."""

    def __init__(self, seed, hq, hkv, page, most, capacity, steps_of):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.page = hq, hkv, page
        batch = len(steps_of[0])
        self.width = -(-capacity // page)
        self.k = torch.full((batch * self.width, page, hkv, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.v = self.k.clone()
        self.cache = pec.PagedCache(self.k, self.v)
        self.table = torch.randperm(batch * self.width, generator=g).view(batch, self.width).to(torch.int32).to(DEV)
        self.weights = [1 + 0.2 * torch.randn(128, generator=g) for _ in range(2)]
        self.angles = angles(capacity)
        self.turn = pec.NormRope(self.angles.to(DEV), *[w.to(DEV) for w in self.weights])
        self.cu = torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
        self.len_k = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.qkv = torch.zeros(most, hq + 2 * hkv, 128, dtype=torch.bfloat16, device=DEV)
        self.q = torch.zeros(most, hq, 128, dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros(hq, most, device=DEV)
        self.ws = torch.empty(pec.pec_paged_workspace_bytes(hq, hkv, batch, most), dtype=torch.uint8, device=DEV)
        self.steps, self.at, self.g = steps_of, [0] * batch, g
        self.fed = [[] for _ in range(batch)]

    def feed(self, new):
        """The next step's inputs into the buffers; rows behind the last sequence hold NaN."""
        rows = sum(new)
        x = torch.full(self.qkv.shape, float("nan"), dtype=torch.bfloat16)
        x[:rows] = torch.randn(rows, *x.shape[1:], generator=self.g).to(torch.bfloat16)
        self.qkv.copy_(x)
        r = 0
        for i, n in enumerate(new):
            self.fed[i].append(x[r:r + n])
            self.at[i] += n
            r += n
        self.cu.copy_(torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32))
        self.len_k.copy_(torch.tensor(self.at, dtype=torch.int32))
        self.out.fill_(3.0)
        self.lse.fill_(3.0)

    def run(self, hints):
        hq, hkv = self.hq, self.hkv
        pec.pec_paged_append(self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:], self.cache, self.table, self.cu, self.len_k,
                             norm_rope=self.turn, q=self.qkv[:, :hq], q_out=self.q)
        pec.pec_attn_paged(self.q, self.cache, self.table, self.cu, self.len_k, *hints, out=self.out, lse=self.lse, workspace=self.ws)

    def check(self, new, what):
        """Against the definitions, from the inputs of all steps so far.  Keys and queries are rounded to bf16 once: the
        reference takes them as the call left them, after holding those to the definition."""
        b = ref.Batch.__new__(ref.Batch)
        b.hq, b.hkv, b.seqs, b.rows = self.hq, self.hkv, list(zip(new, self.at)), sum(new)
        b.cu = self.cu.cpu()
        b.keys, b.values = [], []
        kc, vc, table = self.k.cpu(), self.v.cpu(), self.table.cpu().long()
        for i, t in enumerate(self.at):
            x = torch.cat(self.fed[i])
            pos = torch.arange(t)
            where = table[i][pos // self.page], pos % self.page
            b.keys.append(kc[where])
            b.values.append(vc[where])
            assert torch.equal(b.values[i], x[:, self.hq + self.hkv:])
            ref.assert_rows(b.keys[i], *ref.norm_rope(x[:, self.hq:self.hq + self.hkv], self.weights[1], 1e-6, self.angles, pos), what)
            r0, n = int(b.cu[i]), new[i]
            ref.assert_rows(self.q[r0:r0 + n], *ref.norm_rope(x[t - n:, :self.hq], self.weights[0], 1e-6, self.angles, pos[t - n:]), what)
        ref.assert_attention(self.out, self.lse, ref.attention(b, q=self.q.cpu()), what)
        assert bool((self.out[b.rows:] == 3).all()) and bool((self.lse[:, b.rows:] == 3).all())


STEPS = [[70, 33, 128], [1, 1, 40], [1, 0, 1], [5, 1, 1], [1, 1, 1]]      # prompts, chunks, decode steps and drafted tokens in turn


def test_a_layers_steps_one_behind_the_other():
    layer = Layer(50, 8, 2, 16, 240, 400, STEPS)
    for i, new in enumerate(STEPS):
        layer.feed(new)
        layer.run((max(new), max(layer.at)) if i % 2 else (0, 0))
        layer.check(new, "step %d" % i)


def test_prompts_in_pages_are_prompts_in_a_row():
    """pec_qk_norm_rope and pec_attn_varlen on the same prompts as append and paged attention."""
    layer = Layer(51, 8, 2, 32, 300, 200, [[120, 7, 160]])
    layer.feed([120, 7, 160])
    layer.run((160, 160))
    n = 287
    at = torch.cat([torch.arange(m) for m in (120, 7, 160)]).to(torch.int32).to(DEV)
    q, k = pec.pec_qk_norm_rope(layer.qkv[:n, :8], layer.qkv[:n, 8:10], layer.turn, positions=at)
    assert torch.equal(q, layer.q[:n])
    out, lse = pec.pec_attn_varlen(q, k, layer.qkv[:n, 10:].contiguous(), layer.cu, 160)
    layer.check([120, 7, 160], "paged")
    # both are within two roundings of the weights and one of the result of the same numbers
    assert bool(((out.float() - layer.out[:n].float()).abs() <= 4 * ref.BF16 * (1 + out.float().abs())).all())


@pytest.mark.parametrize("hints", [(1, 60), (1, 4000), (300, 4000)])      # units, steps, steps beside a list (300 packed rows)
def test_captured_steps_work_on_what_the_buffers_hold(hints):
    """Two graphs of one layer through one workspace, replayed in turn with eager work between them; lengths and inputs change."""
    layer = Layer(52, 8, 2, 16, 300, 4000, [[1] * 6])
    layer.feed([3, 7, 1, 9, 4, 2])
    layer.run(hints)                          # (first use outside a capture)
    layer.check([3, 7, 1, 9, 4, 2], "eager")
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            layer.run(hints)
        graphs.append(g)
    for i, new in enumerate([[1] * 6, [2, 0, 1, 1, 5, 1], [1] * 6, [4, 4, 4, 4, 4, 4], [1, 0, 0, 0, 0, 1]]):
        layer.feed(new)
        graphs[i % 2].replay()
        layer.check(new, "replay %d" % i)
        if i == 2:
            layer.feed([1] * 6)
            layer.run((0, 0))
            layer.check([1] * 6, "eager between replays")


@pytest.mark.parametrize("case", HIDDEN, ids=lambda c: c[0])
def test_a_stream_given_keeps_its_workspace(case):
    """What is allocated behind the call on the current stream is not the workspace that the other stream works with."""
    _, seqs, hints = case
    b = ref.Batch(35, 4, 2, 16, seqs, table_extra=BIG // 16)
    alone = attend(b, hints)
    kc, vc, bt, cu, lk = b.to(DEV)
    cache, q, side = pec.PagedCache(kc, vc), b.q.to(DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    n = pec.pec_paged_workspace_bytes(4, 2, len(seqs), b.total)
    out, lse = torch.zeros_like(q), torch.zeros(4, b.total, device=DEV)
    torch.cuda.synchronize()
    for _ in range(10):
        pec.pec_attn_paged(q, cache, bt, cu, lk, *hints, out=out, lse=lse, stream=side)
        torch.full((n,), 255, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        assert torch.equal(out, alone[0]) and torch.equal(lse, alone[1])


@pytest.mark.parametrize("hints", [(1, 60), (16, BIG), (32, BIG), (300, BIG)])
def test_sequences_that_overlap(hints):
    """Offsets that fall again and again, more rows in all than there are packed ones: some result, the rows of no sequence left
    alone, and the next call as ever."""
    seqs = [(300, 400)] + [(0, 60)] * 39
    b = ref.Batch(36, 4, 2, 16, seqs, spare_rows=3, table_extra=BIG // 16)
    right = b.cu
    b.cu = torch.tensor([0, 300] * 20 + [300], dtype=torch.int32)
    attend(b, hints, workspace=torch.full((pec.pec_paged_workspace_bytes(4, 2, 40, b.total),), 255, dtype=torch.uint8, device=DEV))
    b.cu = right
    ref.assert_attention(*attend(b, hints), ref.attention(b), str(hints))


@pytest.mark.parametrize("hints", [(1, BIG), (700, BIG)])      # steps, steps beside a list
def test_as_many_sequences_as_there_may_be(hints):
    """65,536 sequences of one token, appended and looked at: the result is the token's own value, the LSE its score."""
    n, hq, hkv = 65536, 4, 2
    g = torch.Generator().manual_seed(37)
    k, v, q = [torch.randn(n, h, 128, generator=g).to(torch.bfloat16) for h in (hkv, hkv, hq)]
    table = torch.full((n, BIG // 8), -1, dtype=torch.int32, device=DEV)
    table[:, 0] = torch.randperm(n, generator=g).to(torch.int32).to(DEV)
    cache = pec.PagedCache(*[torch.full((n, 8, hkv, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)])
    cu, lk = torch.arange(n + 1, dtype=torch.int32, device=DEV), torch.ones(n, dtype=torch.int32, device=DEV)
    pec.pec_paged_append(k.to(DEV), v.to(DEV), cache, table, cu, lk)
    out, lse = pec.pec_attn_paged(q.to(DEV), cache, table, cu, lk, *hints)
    assert torch.equal(out.cpu(), v.repeat_interleave(hq // hkv, dim=1))      # (a weight of 1 and a sum within 2^-20 of 1)
    product = q.double() * k.repeat_interleave(hq // hkv, dim=1).double() * 128 ** -0.5
    want = product.sum(dim=-1)
    err = (lse.cpu().double().T - want).abs()
    assert bool((err <= 2 * (128 * ref.F32 * product.abs().sum(dim=-1) + 2.0 ** -20) + 2.0 ** -20 * want.abs()).all())


def test_append_in_place():
    """q_out may be a packed q."""
    b = ref.Batch(53, 4, 2, 16, [(5, 30), (1, 8)])
    kc, vc, bt, cu, lk = b.to(DEV)
    table = angles(30)
    q, k, v = b.q.to(DEV), torch.randn(6, 2, 128).to(torch.bfloat16), torch.randn(6, 2, 128).to(torch.bfloat16)
    at = torch.tensor([25, 26, 27, 28, 29, 7])
    got = pec.pec_paged_append(k.to(DEV), v.to(DEV), pec.PagedCache(kc, vc), bt, cu, lk, norm_rope=pec.NormRope(table.to(DEV)), q=q, q_out=q)
    assert got is q
    ref.assert_rows(q, *ref.norm_rope(b.q, None, 0, table, at))


def test_empty_calls():
    b = ref.Batch(54, 4, 2, 16, [(1, 5)])
    kc, vc, bt, cu, lk = b.to(DEV)
    cache = pec.PagedCache(kc, vc)
    none = torch.zeros(0, 4, 128, dtype=torch.bfloat16, device=DEV)
    out, lse = pec.pec_attn_paged(none, cache, bt, cu, lk)
    assert out.shape == (0, 4, 128) and lse.shape == (4, 0)
    pec.pec_paged_append(none[:, :2], none[:, :2], cache, bt, cu, lk)
    assert pec.pec_qk_norm_rope(none, none[:, :2], pec.NormRope())[0].shape == (0, 4, 128)
    no_seq = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    pec.pec_attn_paged(b.q.to(DEV), cache, no_seq, torch.zeros(1, dtype=torch.int32, device=DEV), lk[:0])
