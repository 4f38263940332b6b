"""Calls on a paged cache for the tests: pools and tables, and the operators from their definitions in 64 bits."""
import math

import torch

from paper_2403_18647_amd import binding as B

PAGE = 32
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # a rounding's relative error, at most


def half_step(t):
    return HALF_STEP[t]


def place(slot):
    """Where V's pages hold a slot of a page."""
    s = slot % PAGE
    return s // 4 % 4 * 8 + s // 16 * 4 + s % 4


class Call:
    """Sequences (new, cached) with pages scattered over a pool, and a handle."""

    def __init__(self, seqs, heads, kv, dh, dtype="bf16", spare=0, fill=None, seed=0, max_batch=None, max_ctx=None,
                 extra_pages=3, pages_width=0, n_pages=None, max_rows=None):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.seqs, self.heads, self.kv, self.dh, self.dtype = seqs, heads, kv, dh, TYPES[dtype]
        self.start = [0]
        for n, _ in seqs:
            self.start.append(self.start[-1] + n)
        self.rows = self.start[-1] + spare
        counts = [-(-(n + c) // PAGE) for n, c in seqs]
        self.width = max(max(counts), 1, pages_width)
        self.n_pages = sum(counts) + extra_pages if n_pages is None else n_pages
        ids = torch.randperm(self.n_pages, generator=self.g, device="cuda").int()
        self.pages = torch.full((len(seqs), self.width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(counts):
            self.pages[b, :c] = ids[at:at + c]
            at += c
        self.max_q = max(n for n, _ in seqs)
        self.max_len = max(n + c for n, c in seqs)
        self.paged = B.Paged(B.sdsat_paged_config(
            heads, kv, dh, B.DTYPE_BF16 if dtype == "bf16" else B.DTYPE_FP32, self.n_pages, max_rows or max(1, self.rows),
            max_batch or len(seqs), max_ctx or max(1, self.max_len)))
        self.handle = self.paged.handle
        self.k, self.v = self.paged.pool()
        if fill is None:
            self.k.copy_(self.randn(self.k.shape))
            self.v.copy_(self.randn(self.v.shape))
        else:
            self.k.fill_(fill)
            self.v.fill_(fill)
        self.describe()

    def describe(self):
        t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        self.d_start, self.d_len = t(self.start), t([c for _, c in self.seqs])
        self.batch = B.paged_batch(self.d_start, self.d_len, self.pages, self.rows, self.max_q, self.max_len)

    def randn(self, shape, dtype=None, scale=1.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * scale).to(dtype or self.dtype)

    def slots(self, b, first, last):
        """Pages and places of slots first .. last - 1 of sequence b."""
        s = torch.arange(first, last, device="cuda")
        return self.pages[b].long()[s // PAGE], s % PAGE

    def put(self, b, first, k, v):
        """Rows k and v [slots, kv, dh] to the slots from `first` on."""
        page, at = self.slots(b, first, first + k.shape[0])
        self.k[page, :, at] = k.to(self.dtype)
        self.v[page, :, :, place(at)] = v.to(self.dtype)

    def get(self, b, first, last):
        page, at = self.slots(b, first, last)
        return self.k[page, :, at], self.v[page, :, :, place(at)]

    def attend(self, q, mask=None, window=0, scale=0.0, out=None):
        out = torch.zeros_like(q) if out is None else out
        B.sdsat_paged_attention(self.handle, self.batch, self.k, self.v, q, mask, window, scale, out)
        return out

    def visible(self, b, mask, window):
        """[new, new + cached] truth of sequence b."""
        n, c = self.seqs[b]
        slot = torch.arange(n + c, device="cuda")[None]
        at = torch.arange(c, c + n, device="cuda")[:, None]
        if mask is None:
            see = slot <= at
            return see & (slot > at - window) if window else see
        bits = mask[self.start[b]:self.start[b] + n, None] >> (slot - c).clamp(0, 63) & 1
        return (slot < c) | (bits == 1)

    def expected(self, q, mask=None, window=0, scale=0.0, u_out=None):
        """The attention in 64 bits, and how far the kernel's may be from it.

        Half a step of the output; half a step of each weight (bf16; fp32 weights are not rounded); the scores' error, dh
        roundings of sums of |q| |k| (taken twice, for the order in which the cores add) on an exponent that the maximum
        shares, so 2 scores'; a rounding per slot and 64 more for sums, rescalings, joins and the exponential."""
        scale = scale or 1 / math.sqrt(self.dh)
        per = self.heads // self.kv
        out = torch.zeros((q.shape[0], self.heads, self.dh), dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(out)
        qd = q.double().view(q.shape[0], self.heads, self.dh)
        u = half_step(self.dtype) if u_out is None else u_out
        for b, (n, c) in enumerate(self.seqs):
            if n == 0:
                continue
            see = self.visible(b, mask, window)
            kb, vb = (t.double() for t in self.get(b, 0, n + c))
            r = slice(self.start[b], self.start[b] + n)
            for h in range(self.heads):
                k = torch.where(see.any(0)[:, None], kb[:, h // per], 0.0)
                v = torch.where(see.any(0)[:, None], vb[:, h // per], 0.0)
                s = (torch.matmul(qd[r, h], k.t().contiguous()) * scale).masked_fill(~see, -math.inf)
                size = torch.matmul(qd[r, h].abs(), k.abs().t().contiguous()).masked_fill(~see, 0.0).amax(1) * scale
                top = s.amax(1, keepdim=True)
                w = torch.where(see, torch.exp(s - torch.where(top.isinf(), 0.0, top)), 0.0)
                den = w.sum(1, keepdim=True)
                w = w / torch.where(den == 0, 1.0, den)
                o = torch.matmul(w, v)
                a = torch.matmul(w, v.abs())
                rel = 2 * (2 * self.dh + 4) * 2.0 ** -24 * size + (n + c + 64) * 2.0 ** -23
                rel = rel + (half_step(self.dtype) if self.dtype == torch.bfloat16 else 0.0)
                out[r, h] = o
                tol[r, h] = u * o.abs() + rel[:, None] * a * (1 + u) + 1e-30
        return out.view(q.shape[0], -1), tol.view(q.shape[0], -1)


def assert_within(got, want, tol, what=""):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}, "
                           f"worst {float((off / tol).nan_to_num(math.inf).max()):.3g} of what is allowed")
    return float((off / tol).max()) if off.numel() else 0.0


def tree_mask(n, width=2):
    k = (n - 1) // width
    mask = [1] + [(1 << (j + 1)) - 1 for j in range(1, k + 1)]
    for j in range(1, k + 1):
        for _ in range(width - 1):
            mask.append(((1 << j) - 1) | (1 << len(mask)))
    return mask


def int64(values):
    """64-bit patterns as a device tensor."""
    return torch.tensor([v - (1 << 64) if v >> 63 else v for v in values], dtype=torch.int64, device="cuda")
