"""Operators of a layer's step between the projection of queries, keys and values and the output projection, where a server
keeps the keys and values in pages: norms of queries and keys with the rotation of positions (`rope`), the same with the new
keys and values going into the paged cache (`append`), and attention of every sequence's new tokens over its pages (`attn`).

`listed()` are the cases that are timed, `draw()` makes more of the same ranges, `prepare()` makes what a server holds ahead of
the call, `run()` makes the call (the framework's with `own`, elementary torch operations in 32 bits without), `work()` counts
what it cannot do without, `exact()` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DIM = 128                   # head dim of the framework
EPS = 1e-6
LARGEST_FLOPS = 8.5e12      # no drawn case costs more than the largest listed ones
LARGEST_BYTES = 2.2e9


# ---- cases

def _attn(name, hq, hkv, page, lengths, steps=0, step_q=1, ctx=0, spread=False, chunks=0, chunk_q=0, chunk_ctx=0, by_head=False,
          causal=True):
    """`steps` sequences with `step_q` new tokens on about `ctx` cached ones (spread: log-normal around it, up to 12 times as
    many), then `chunks` sequences with about `chunk_q` new tokens behind about `chunk_ctx` cached ones.  `lengths` seeds them."""
    return {"op": "attn", "name": name, "hq": hq, "hkv": hkv, "page": page, "lengths": lengths, "steps": steps, "step_q": step_q,
            "ctx": ctx, "spread": spread, "chunks": chunks, "chunk_q": chunk_q, "chunk_ctx": chunk_ctx, "by_head": by_head,
            "causal": causal}


def _append(name, hq, hkv, page, lengths, norm, rotary, interleaved, **seqs):
    c = _attn(name, hq, hkv, page, lengths, **seqs)
    c.update(op="append", norm=norm, rotary=rotary, interleaved=interleaved)
    return c


def _rope(name, tokens, hq, hkv, norm, rotary, interleaved, first, packed):
    """`first`: position of the first token, 0 and on; negative: every token has a position of its own.  `packed`: q and k are
    parts of one projection's output, [tokens, hq + 2 hkv, 128]."""
    return {"op": "rope", "name": name, "tokens": tokens, "hq": hq, "hkv": hkv, "norm": norm, "rotary": rotary,
            "interleaved": interleaved, "first": first, "packed": packed}


def listed():
    return [
        # one decode step of a nearly idle server: all latency
        _attn("attn_step_few", 32, 8, 16, 11, steps=4, ctx=600),
        # one decode step of a busy one, contexts as the short prompts of the paper's trace
        _attn("attn_step_batch", 32, 8, 16, 12, steps=64, ctx=700, spread=True),
        # decode steps of long requests, many heads, large pages
        _attn("attn_step_long", 64, 8, 256, 13, steps=4, ctx=131072),
        # five drafted tokens of every sequence looked at together
        _attn("attn_verify", 64, 8, 32, 14, steps=24, step_q=5, ctx=12000),
        # one chunk of a long prompt, small enough not to hold up the decode steps beside it
        _attn("attn_chunk_512", 32, 8, 64, 15, chunks=1, chunk_q=512, chunk_ctx=30000),
        # a chunk as large as the segments of the sequence-parallel prefill
        _attn("attn_chunk_8k", 32, 8, 64, 16, chunks=1, chunk_q=8192, chunk_ctx=57000),
        # short prompts without a prefix beside decode steps, cache laid out by heads
        _attn("attn_mixed", 32, 8, 16, 17, steps=24, ctx=3500, spread=True, chunks=6, chunk_q=1100, chunk_ctx=0, by_head=True),
        # a step's new keys and values, and its queries
        _append("append_step", 32, 8, 16, 21, False, 128, False, steps=64, ctx=450),
        # chunks of three prompts of a model with normed queries and keys
        _append("append_chunks", 32, 8, 64, 22, True, 128, True, chunks=3, chunk_q=2700, chunk_ctx=5000, by_head=True),
        # single tokens of several sequences
        _rope("rope_step", 48, 32, 8, True, 128, False, -1, True),
        # a ring member's segment of 16,384 tokens with 64 heads
        _rope("rope_segment", 16384, 64, 8, True, 128, False, 49152, True),
        # a prompt of a model that rotates a part of each head, as many key heads as query heads
        _rope("rope_partial", 1931, 8, 8, False, 64, True, 0, False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 5, 8])
        page = rng.choice([16, 32, 64, 128, 256])
        lengths = rng.randrange(1 << 20)
        by_head = rng.random() < 0.3
        kind = rng.choice(["step", "step", "verify", "chunk", "chunk", "mixed", "append", "append", "rope", "rope"])
        if kind == "step":
            c = _attn("", hq, hkv, page, lengths, steps=_log(rng, 1, 128), ctx=_log(rng, 64, 131072), spread=rng.random() < 0.5,
                      by_head=by_head)
        elif kind == "verify":
            c = _attn("", hq, hkv, page, lengths, steps=_log(rng, 1, 48), step_q=rng.randint(2, 9), ctx=_log(rng, 64, 16384),
                      by_head=by_head)
        elif kind == "chunk":
            c = _attn("", hq, hkv, page, lengths, chunks=rng.randint(1, 4), chunk_q=_log(rng, 64, 8192), chunk_ctx=_log(rng, 1, 57000),
                      by_head=by_head, causal=rng.random() < 0.85)
        elif kind == "mixed":
            c = _attn("", hq, hkv, page, lengths, steps=_log(rng, 1, 48), ctx=_log(rng, 64, 16384), spread=True,
                      chunks=rng.randint(1, 6), chunk_q=_log(rng, 32, 2048), chunk_ctx=rng.choice([0, _log(rng, 1, 8192)]),
                      by_head=by_head)
        elif kind == "append":
            what = dict(norm=rng.random() < 0.5, rotary=rng.choice([0, 32, 64, 128, 128]), interleaved=rng.random() < 0.4,
                        by_head=by_head)
            if rng.random() < 0.5:
                c = _append("", hq, hkv, page, lengths, steps=_log(rng, 1, 128), ctx=_log(rng, 16, 500), **what)
            else:
                c = _append("", hq, hkv, page, lengths, chunks=rng.randint(1, 4), chunk_q=_log(rng, 16, 4096),
                            chunk_ctx=_log(rng, 1, 4096), **what)
        else:
            c = _rope("", _log(rng, 1, 16384), hq, hkv, rng.random() < 0.5, rng.choice([32, 64, 128, 128]), rng.random() < 0.4,
                      rng.choice([-1, 0, rng.randint(1, 49152)]), rng.random() < 0.6)
        w = work(c)
        if w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES:
            del c["name"]
            return c


def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of every sequence."""
    rng = random.Random(case["lengths"])
    new, total = [], []
    for _ in range(case["steps"]):
        if case["spread"]:
            n = int(round(case["ctx"] * math.exp(1.27 * rng.gauss(0.0, 1.0))))
            n = max(1, min(n, 12 * case["ctx"]))
        else:
            n = rng.randint(max(1, int(0.7 * case["ctx"])), case["ctx"])
        new.append(case["step_q"])
        total.append(n + case["step_q"])
    for _ in range(case["chunks"]):
        n = case["chunk_q"] if case["chunks"] == 1 else rng.randint(max(1, case["chunk_q"] // 2), case["chunk_q"])
        ctx = rng.randint(int(0.9 * case["chunk_ctx"]), case["chunk_ctx"]) if case["chunk_ctx"] else 0
        new.append(n)
        total.append(n + ctx)
    order = list(range(len(new)))
    rng.shuffle(order)
    return [new[i] for i in order], [total[i] for i in order]


def _positions(case, tokens):
    """Positions of the tokens of a `rope` case without a common start."""
    rng = random.Random(tokens)
    return [rng.randrange(8192) for _ in range(tokens)]


# ---- inputs

def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _table(positions, rotary):
    """Cosines, then sines, of every position's angles, from 64 bits."""
    half = rotary // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * freq[None]
    return torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    host = random.Random(seed)
    hq, hkv = case["hq"], case["hkv"]
    st = {"case": dict(case)}
    if case["op"] == "rope":
        n = case["tokens"]
        last = (8191 if case["first"] < 0 else case["first"] + n - 1) if n else 0
        if case["first"] < 0:
            st["positions"] = torch.tensor(_positions(case, n), dtype=torch.int32, device=DEV)
        else:
            st["positions"] = None
    else:
        new, total = _lengths(case)
        n, last = sum(new), max(total) - 1
    if case["op"] != "attn":
        qkv = _randn(gen, n, hq + 2 * hkv, DIM)
        parts = [qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]]
        if case["op"] == "rope" and not case["packed"]:
            parts = [t.contiguous() for t in parts]
        st["q"], st["k"], st["v"] = parts
        st["table"] = _table(last + 1, case["rotary"]) if case["rotary"] else None
        st["q_weight"] = 1 + 0.2 * torch.randn(DIM, generator=gen, device=DEV) if case["norm"] else None
        st["k_weight"] = 1 + 0.2 * torch.randn(DIM, generator=gen, device=DEV) if case["norm"] else None
        st["q_out"] = torch.empty(n, hq, DIM, dtype=torch.bfloat16, device=DEV)
    if case["op"] == "rope":
        st["k_out"] = torch.empty(n, hkv, DIM, dtype=torch.bfloat16, device=DEV)
        return st
    page, by_head = case["page"], case["by_head"]
    need = [-(-t // page) for t in total]
    n_pages = sum(need) + max(2, sum(need) // 16)
    shape = (n_pages, hkv, page, DIM) if by_head else (n_pages, page, hkv, DIM)
    st["k_cache"], st["v_cache"] = [t.transpose(1, 2) if by_head else t for t in (_randn(gen, *shape), _randn(gen, *shape))]
    numbers = list(range(n_pages))
    host.shuffle(numbers)
    rows, at = [], 0
    for m in need:      # behind a sequence's last page the table holds whatever was there
        rows.append(numbers[at:at + m] + [host.randrange(n_pages) for _ in range(max(need) - m)])
        at += m
    st["block_table"] = torch.tensor(rows, dtype=torch.int32, device=DEV)
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    st["cu_q"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    st["len_k"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    st["new"], st["total"] = new, total
    if case["op"] == "attn":
        st["q"] = _randn(gen, n, hq, DIM)
        st["out"] = torch.empty(n, hq, DIM, dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty(hq, n, dtype=torch.float32, device=DEV)
    return st


# ---- one pass

def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "append": _plain_append, "rope": _plain_rope}[state["case"]["op"]](state)


def _run_own(st):
    from paper_2409_15104_amd import binding as pec

    case = st["case"]
    if "handles" not in st:     # made once by a server: the model's norms and rotation, the cache, a workspace
        norm_rope = cache = workspace = None
        if case["op"] != "attn":
            norm_rope = pec.NormRope(st["table"], st["q_weight"], st["k_weight"], eps=EPS, interleaved=case["interleaved"])
        if case["op"] != "rope":
            cache = pec.PagedCache(st["k_cache"], st["v_cache"])
        if case["op"] == "attn":
            workspace = torch.empty(pec.pec_paged_workspace_bytes(case["hq"], case["hkv"], len(st["new"]), sum(st["new"])),
                                    dtype=torch.uint8, device=DEV)
        st["handles"] = norm_rope, cache, workspace
    norm_rope, cache, workspace = st["handles"]
    if case["op"] == "rope":
        pec.pec_qk_norm_rope(st["q"], st["k"], norm_rope, positions=st["positions"], pos0=max(0, case["first"]),
                             q_out=st["q_out"], k_out=st["k_out"])
        return st["q_out"], st["k_out"]
    if case["op"] == "append":
        pec.pec_paged_append(st["k"], st["v"], cache, st["block_table"], st["cu_q"], st["len_k"], norm_rope=norm_rope,
                             q=st["q"], q_out=st["q_out"])
        return st["q_out"], st["k_cache"], st["v_cache"]
    pec.pec_attn_paged(st["q"], cache, st["block_table"], st["cu_q"], st["len_k"], max_len_q=max(st["new"]),
                       max_len_k=max(st["total"]), causal=case["causal"], out_dtype=st["out"].dtype, out=st["out"],
                       lse=st["lse"], workspace=workspace)
    return st["out"], st["lse"]


def _plain_norm_rope(x, weight, table, positions, interleaved):
    """[tokens, heads, 128] bf16 -> fp32, normed if there is a weight and rotated if there is a table."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight
    if table is None:
        return x
    half = table.shape[1] // 2
    rows = table[positions]
    c, s = rows[:, None, :half], rows[:, None, half:]
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _plain_rope(st):
    case = st["case"]
    at = st["positions"]
    if at is None:
        at = torch.arange(case["first"], case["first"] + case["tokens"], device=DEV)
    return tuple(_plain_norm_rope(x, w, st["table"], at, case["interleaved"]).to(torch.bfloat16)
                 for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])))


def _plain_append(st):
    case, page = st["case"], st["case"]["page"]
    cu, len_k = st["cu_q"].long(), st["len_k"].long()
    token = torch.arange(st["q"].shape[0], device=DEV)
    seq = torch.bucketize(token, cu[1:], right=True)
    at = len_k[seq] - cu[seq + 1] + token
    number, slot = st["block_table"].long()[seq, at // page], at % page
    q, k = [_plain_norm_rope(x, w, st["table"], at, case["interleaved"]).to(torch.bfloat16)
            for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"]))]
    st["k_cache"][number, slot] = k
    st["v_cache"][number, slot] = st["v"]
    return q, st["k_cache"], st["v_cache"]


def _plain_attn(st):
    case = st["case"]
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    g, scale = hq // hkv, 1.0 / math.sqrt(DIM)
    out = torch.empty_like(st["out"])
    lse = torch.empty_like(st["lse"])
    q0 = 0
    for b, (nq, nk) in enumerate(zip(st["new"], st["total"])):
        numbers = st["block_table"][b, :-(-nk // page)].long()
        k, v = [c[numbers].flatten(0, 1)[:nk].float().transpose(0, 1).contiguous() for c in (st["k_cache"], st["v_cache"])]
        kt = k.transpose(1, 2).contiguous()                                     # [hkv, 128, nk]
        rows = max(1, min(nq, (1 << 29) // (hq * nk)))                          # as many queries at a time as 2 GiB of scores hold
        for r in range(0, nq, rows):
            n = min(rows, nq - r)
            q = st["q"][q0 + r:q0 + r + n].float().view(n, hkv, g, DIM).permute(1, 2, 0, 3).reshape(hkv, g * n, DIM)
            s = torch.matmul(q, kt).mul_(scale).view(hkv, g, n, nk)
            if case["causal"]:
                hidden = torch.arange(nk, device=DEV)[None] > (nk - nq + r + torch.arange(n, device=DEV))[:, None]
                s.masked_fill_(hidden, -math.inf)
            top = s.amax(dim=-1, keepdim=True)
            s = s.sub_(top).exp_()
            den = s.sum(dim=-1, keepdim=True)
            o = torch.matmul(s.view(hkv, g * n, nk), v).view(hkv, g, n, DIM) / den
            out[q0 + r:q0 + r + n] = o.permute(2, 0, 1, 3).reshape(n, hq, DIM).to(out.dtype)
            lse[:, q0 + r:q0 + r + n] = (top + den.log()).view(hq, n)
        q0 += nq
    return out, lse


# ---- counts and the definition

def _elements(case):
    """bf16 values of queries, of keys, flop per value of a head row."""
    per = (4.0 if case["norm"] else 0.0) + (3.0 * case["rotary"] / DIM)
    return case["hq"] * DIM, case["hkv"] * DIM, per


def work(case):
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "rope":
        n = case["tokens"]
        rows = n if case["first"] >= 0 else len(set(_positions(case, n)))
        eq, ek, per = _elements(case)
        return {"bytes": 4.0 * n * (eq + ek) + 4.0 * rows * case["rotary"], "flops": n * (eq + ek) * per}
    new, total = _lengths(case)
    n = sum(new)
    if case["op"] == "append":
        eq, ek, per = _elements(case)
        rows = len({t - m + i for m, t in zip(new, total) for i in range(m)})
        return {"bytes": 4.0 * n * (eq + 2 * ek) + 4.0 * rows * case["rotary"], "flops": n * (eq + ek) * per}
    pairs = sum(m * (t - m) + m * (m + 1) // 2 if case["causal"] else m * t for m, t in zip(new, total))
    keys = 4.0 * DIM * hkv * sum(total)
    return {"bytes": keys + n * hq * (4.0 * DIM + 4.0), "flops": 4.0 * DIM * hq * pairs}


def exact(case, seed):
    """From the definitions, in 64 bits: every head on its own, positions and pages looked up on the host."""
    st = prepare(case, seed)
    f64 = torch.float64

    def turned(x, weight, at):
        y = x.to(f64)
        if weight is not None:
            y = y / ((y ** 2).sum(-1, keepdim=True) / DIM + EPS).sqrt() * weight.to(f64)
        if st["table"] is None:
            return y
        r = case["rotary"]
        z = torch.complex(*[t.to(f64) for t in (st["table"][at, :r // 2], st["table"][at, r // 2:])])[:, None]
        i = torch.arange(r // 2, device=DEV)
        lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
        w = torch.complex(y[..., lo], y[..., hi]) * z
        y[..., lo], y[..., hi] = w.real, w.imag
        return y

    if case["op"] == "rope":
        n = case["tokens"]
        at = _positions(case, n) if case["first"] < 0 else range(case["first"], case["first"] + n)
        at = torch.tensor(list(at), device=DEV)
        return turned(st["q"], st["q_weight"], at), turned(st["k"], st["k_weight"], at)
    page = case["page"]
    table = st["block_table"].tolist()
    if case["op"] == "append":
        at = [t - m + i for m, t in zip(st["new"], st["total"]) for i in range(m)]
        where = [(table[b][p // page], p % page) for b, (m, t) in enumerate(zip(st["new"], st["total"])) for p in range(t - m, t)]
        pages, slots = torch.tensor(where, device=DEV).T
        at = torch.tensor(at, device=DEV)
        k, v = st["k_cache"].to(f64), st["v_cache"].to(f64)
        k.index_put_((pages, slots), turned(st["k"], st["k_weight"], at))
        v.index_put_((pages, slots), st["v"].to(f64))
        return turned(st["q"], st["q_weight"], at), k, v
    hq, hkv = case["hq"], case["hkv"]
    n = sum(st["new"])
    out = torch.empty(n, hq, DIM, dtype=f64, device=DEV)
    lse = torch.empty(hq, n, dtype=f64, device=DEV)
    q0 = 0
    for b, (m, t) in enumerate(zip(st["new"], st["total"])):
        pages = torch.tensor(table[b][:-(-t // page)], device=DEV)
        for h in range(hkv):
            k = st["k_cache"][pages, :, h].reshape(-1, DIM)[:t].to(f64)
            v = st["v_cache"][pages, :, h].reshape(-1, DIM)[:t].to(f64)
            kt = k.t().contiguous()
            for head in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                step = max(1, (1 << 27) // t)
                for r in range(0, m, step):
                    e = min(m, r + step)
                    s = (st["q"][q0 + r:q0 + e, head].to(f64) @ kt) / DIM ** 0.5
                    if case["causal"]:
                        last = torch.arange(t - m + r, t - m + e, device=DEV)
                        s[torch.arange(t, device=DEV)[None, :] > last[:, None]] = -math.inf
                    lse[head, q0 + r:q0 + e] = torch.logsumexp(s, dim=-1)
                    out[q0 + r:q0 + e, head] = torch.softmax(s, dim=-1) @ v
        q0 += m
    return out, lse
