"""Plain 64-bit definition of the 4-bit format of a paged cache, on the CPU, and batches whose cache is in it."""
import torch

from paged_reference import DIM, Batch

GROUP = 32
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """x [..., 128] bf16 -> (codes uint8 [..., 64], scale bytes uint8 [..., 4]) by the definition: the scale from the group's largest
    magnitude, then the nearest level, the even one of two that are as near."""
    g = x.double().unflatten(-1, (-1, GROUP))
    bad = ~g.isfinite().all(dim=-1)
    g = torch.where(bad[..., None], torch.zeros_like(g), g)
    top = g.abs().amax(dim=-1)
    frac, e = torch.frexp(top)                       # top = (2 frac) 2^(e - 1)
    e = torch.where(2 * frac >= 1.75, e - 2, e - 3)
    e = torch.where(top == 0, torch.full_like(e, -125), e).clamp(-125, 125)
    y = torch.ldexp(g, -e[..., None].double())
    dist = (y.abs()[..., None] - LEVELS).abs()
    least = dist.amin(dim=-1, keepdim=True)
    even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    pick = (dist[..., even_first] == least).int().argmax(dim=-1)
    code = even_first[pick] + 8 * torch.signbit(x).unflatten(-1, (-1, GROUP)).long()
    code = torch.where(bad[..., None], torch.zeros_like(code), code).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), scale.to(torch.uint8)


def values(codes, scale):
    """What codes [..., 64] and scale bytes [..., 4] stand for, in 64 bits."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    y = torch.where(c >= 8, -LEVELS[c & 7], LEVELS[c & 7]).unflatten(-1, (-1, GROUP))
    f = torch.ldexp(torch.ones((), dtype=torch.float64), scale.double() - 127)
    f = torch.where(scale == 255, torch.full_like(f, float("nan")), f)
    return (y * f[..., None]).flatten(-2)


class MxBatch(Batch):
    """A Batch whose cache is in 4 bits: k, v become codes [pages, slots, heads, 64], k_scale, v_scale bytes [pages, heads, 4, slots] (NaN
    wherever no token of a sequence is), and keys, values what is held of them, so that the definitions of a Batch's attention go for it."""

    def __init__(self, *args, **kw):
        self.k_scale = None
        super().__init__(*args, **kw)
        n, page, hkv, _ = self.k.shape
        self.k = torch.randint(0, 256, (n, page, hkv, DIM // 2), dtype=torch.uint8, generator=torch.Generator().manual_seed(args[0]))
        self.v = self.k.clone()
        self.k_scale = torch.full((n, hkv, DIM // GROUP, page), 255, dtype=torch.uint8)
        self.v_scale = self.k_scale.clone()
        self.raw = [(k, v) for k, v in zip(self.keys, self.values)]      # before they were rounded
        for b in range(len(self.seqs)):
            self.put(b)

    def where(self, b, first=0):
        pos = torch.arange(first, self.seqs[b][1])
        return self.table[b].long()[pos // self.page], pos % self.page

    def put(self, b):
        if self.k_scale is None:      # the base class's own call
            return
        for held, codes, scales in ((self.keys, self.k, self.k_scale), (self.values, self.v, self.v_scale)):
            page, slot = self.where(b)
            c, s = quantise(held[b])
            codes[page, slot] = c
            scales[page, :, :, slot] = s
            held[b] = values(c, s)

    def to(self, device, by_head=False):
        """((k, v, k_scale, v_scale) in the asked layout, table, cu, len_k) on the device."""
        lay = (lambda t: t.transpose(1, 2).contiguous().to(device).transpose(1, 2)) if by_head else (lambda t: t.to(device))
        return ((lay(self.k), lay(self.v), self.k_scale.to(device), self.v_scale.to(device)), self.table.to(device), self.cu.to(device),
                self.len_k.to(device))
