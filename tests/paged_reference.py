"""Plain 64-bit definitions of the paged operators, on the CPU, and batches to try them on."""
import math

import numpy as np
import torch

DIM = 128
BF16, F32 = 2.0 ** -8, 2.0 ** -24       # half a step of the type, relative to the value


def norm_rope(x, weight=None, eps=0.0, cos_sin=None, positions=None, interleaved=False):
    """x [tokens, heads, 128] -> (result in 64 bits, what its rounding errors in fp32 scale with)."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(dim=-1, keepdim=True) + eps) * weight.double()
    size = y.abs()
    if cos_sin is not None:
        half = cos_sin.shape[1] // 2
        rows = cos_sin.double()[positions.long().clamp(0, cos_sin.shape[0] - 1)]
        c, s = rows[:, None, :half], rows[:, None, half:]
        lo = torch.arange(half) * 2 if interleaved else torch.arange(half)
        hi = lo + (1 if interleaved else half)
        a, b = y[..., lo].clone(), y[..., hi].clone()
        y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
        size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return y, size


def assert_rows(got, ref, size, what=""):
    """One rounding to bf16, and in fp32 three products and sums behind a norm of 128 squares: under 2^-24 x (128 / 2 + 8) of it."""
    err = (got.double().cpu() - ref).abs()
    ok = err <= BF16 * ref.abs() + 80 * F32 * size
    assert bool(ok.all()), "%s: off by %.3g at %s" % (what, float(err.max()), np.argwhere(~ok.numpy())[:3].tolist())


class Batch:
    """Sequences [(new tokens, tokens in all)] in a paged cache on the CPU: pages dealt out in random order, NaN wherever no
    token of a sequence is, page numbers that name no page behind every sequence's last one."""

    def __init__(self, seed, hq, hkv, page, seqs, spare_rows=0, spare_pages=3, table_extra=2, wild=True):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.page, self.seqs = hq, hkv, page, seqs
        need = [-(-max(t, 0) // page) for _, t in seqs]
        self.n_pages = sum(need) + spare_pages
        order = torch.randperm(self.n_pages, generator=g).tolist()
        width = max(need, default=0) + table_extra
        self.table = torch.full((len(seqs), width), 0, dtype=torch.int32)
        if wild:
            self.table[:, 0::2], self.table[:, 1::2] = -5, 2 ** 31 - 1
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.cu = torch.tensor([0] + np.cumsum([n for n, _ in seqs]).tolist(), dtype=torch.int32)
        self.len_k = torch.tensor([t for _, t in seqs], dtype=torch.int32)
        self.rows = int(self.cu[-1])
        self.total = self.rows + spare_rows
        rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
        self.q = rnd(self.total, hq, DIM)
        self.k = torch.full((self.n_pages, page, hkv, DIM), float("nan"), dtype=torch.bfloat16)
        self.v = self.k.clone()
        self.keys, self.values = [], []
        for b, (_, t) in enumerate(seqs):
            self.keys.append(rnd(t, hkv, DIM))
            self.values.append(rnd(t, hkv, DIM))
            self.put(b)

    def put(self, b):
        """The sequence's keys and values into its pages."""
        t = self.seqs[b][1]
        pos = torch.arange(t)
        where = self.table[b].long()[pos // self.page], pos % self.page
        self.k[where], self.v[where] = self.keys[b], self.values[b]

    def to(self, device, by_head=False):
        """(cache tensors in the asked layout, table, cu, len_k) on the device."""
        lay = (lambda t: t.transpose(1, 2).contiguous().to(device).transpose(1, 2)) if by_head else (lambda t: t.to(device))
        return lay(self.k), lay(self.v), self.table.to(device), self.cu.to(device), self.len_k.to(device)


def attention(batch, causal=True, scale=None, q=None):
    """Per definition, keys that a row does not see left out: (out [rows, hq, 128], lse [hq, rows], A, S): A = the weighted mean
    of |V|, S = the largest sum of |q k| scale of a row, which the errors scale with."""
    scale = scale or 1 / math.sqrt(DIM)
    q = batch.q if q is None else q
    g = batch.hq // batch.hkv
    out = torch.zeros(batch.rows, batch.hq, DIM, dtype=torch.float64)
    lse = torch.full((batch.hq, batch.rows), -math.inf, dtype=torch.float64)
    a, s_abs = torch.zeros_like(out), torch.zeros_like(lse)
    for b, (n, t) in enumerate(batch.seqs):
        if n == 0 or t == 0:
            continue
        r0 = int(batch.cu[b])
        last = torch.arange(t - n, t) if causal else torch.full((n,), t - 1)
        hidden = torch.arange(t)[None] > last[:, None]
        some = last >= 0
        for h in range(batch.hkv):
            k, v = batch.keys[b][:, h].double(), batch.values[b][:, h].double()
            for head in range(h * g, (h + 1) * g):
                x = q[r0:r0 + n, head].double()
                s = (x @ k.T * scale).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(s, dim=-1)
                w = torch.exp(s - torch.where(some, l, torch.zeros_like(l))[:, None])
                clean = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)
                o = w @ clean
                bad = ~v.isfinite()
                for j in bad.any(dim=1).nonzero().flatten().tolist():      # only rows that see such a value are touched by it
                    sees = ~hidden[:, j]
                    o[sees] += torch.where(bad[j], v[j] * 1.0, torch.zeros(DIM, dtype=torch.float64))
                out[r0:r0 + n, head] = torch.where(some[:, None], o, torch.zeros_like(o))
                lse[head, r0:r0 + n] = l
                a[r0:r0 + n, head] = w @ clean.abs()
                s_abs[head, r0:r0 + n] = (x.abs() @ k.abs().T * scale).masked_fill(hidden, 0).amax(dim=-1)
    return out, lse, a, s_abs


def assert_attention(out, lse, ref, what="", plain=False):
    """Scores are sums of 128 products in fp32: off by 128 x 2^-24 of the sum of their sizes at most, and by a few 2^-24 more for
    scale, exponential and logarithm.  A weight is off by that, relative to itself, and rounded to bf16 once (not by the plain
    kernel); sums over n keys in fp32, in blocks, add under 2^-16.  A bf16 result is rounded once more."""
    o_ref, l_ref, a, s_abs = ref
    rows = o_ref.shape[0]
    o, l = out[:rows].double().cpu(), lse[:, :rows].double().cpu()
    tol_s = 2.0 ** -17 * s_abs + 2.0 ** -20
    fin = l_ref.isfinite()
    assert torch.equal(l.isfinite(), fin) and bool((l[~fin] == -math.inf).all()), "%s: -inf pattern of lse" % what
    err = (l - l_ref).abs()[fin]
    assert bool((err <= (2 * tol_s + 2.0 ** -20 * l_ref.abs())[fin]).all()), "%s: lse off by %.3g" % (what, float(err.max()))
    tol = a * (2 * tol_s.T[..., None] + 2.0 ** -16 + (0 if plain else BF16)) + (BF16 * o_ref.abs() if out.dtype == torch.bfloat16 else 0) + 1e-30
    ok_ref = o_ref.isfinite()
    assert torch.equal(o.isfinite(), ok_ref), "%s: finite pattern of out" % what
    err = (o - o_ref).abs()
    bad = (err > tol) & ok_ref
    assert not bool(bad.any()), "%s: out off by %.3g (%.3g allowed) at %s" % (
        what, float(err[bad].max()), float(tol[bad].min()), bad.nonzero()[:3].tolist())
    assert bool((o[~fin.T] == 0).all()), what        # rows without a key are exactly zero
