"""The paged cache and the attention over it in 64 bits, and batches for their tests."""
import math

import torch

from paper_2510_05528_b200 import binding as Bd

DEV = "cuda:0"
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def to_int8(x):
    """int8 rows and fp32 scales; in 64 bits the quotient of two numbers of 24 bits stays on its side of a half."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, torch.round(127 * x / torch.where(top > 0, top, 1.0)), 0.0)
    return q.to(torch.int8), (top[..., 0] / 127).float()


class Case:
    """A cache in some layout with pages in any order, and a batch of (new rows, positions) on it."""

    def __init__(self, sizes, *, kv_heads=2, dim=128, page=16, layout="heads", seed=0, spare=3, dev=DEV):
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        self.gen, self.sizes, self.kv_heads, self.dim, self.page, self.dev = gen, sizes, kv_heads, dim, page, dev
        need = [-(-length // page) for _, length in sizes]
        n = sum(need) + spare
        order = torch.randperm(n, generator=gen, device=dev).int()
        if layout == "heads":                         # [pages, heads, slots]
            values, scales = [torch.empty(n, kv_heads, page, dim, dtype=torch.int8, device=dev) for _ in "kv"], [torch.empty(n, kv_heads, page, device=dev) for _ in "kv"]
        elif layout == "slots":                       # [pages, slots, heads]
            values, scales = [torch.empty(n, page, kv_heads, dim, dtype=torch.int8, device=dev).transpose(1, 2) for _ in "kv"], [torch.empty(n, page, kv_heads, device=dev).transpose(1, 2) for _ in "kv"]
        else:                                         # keys and values side by side, rows of a wider array, pages innermost but one
            both = torch.empty(kv_heads, page, n, 2, dim + 16, dtype=torch.int8, device=dev).permute(2, 0, 1, 3, 4)
            values = [both[..., i, :dim] for i in (0, 1)]
            scales = [torch.empty(kv_heads, n, page, 2, device=dev)[..., i].transpose(0, 1) for i in (0, 1)]
        for t in values:
            t.copy_(torch.randint(-127, 128, t.shape, generator=gen, device=dev))
        for t in scales:
            t.copy_(torch.exp(torch.randn(t.shape, generator=gen, device=dev)) / 100)
        self.k, self.v, self.k_scale, self.v_scale = *values, *scales
        self.pages = torch.full((len(sizes), max(need + [1])), -7, dtype=torch.int32, device=dev)       # (behind a sequence's pages: never read)
        at = 0
        for b, m in enumerate(need):
            self.pages[b, :m] = order[at:at + m]
            at += m
        self.lengths = torch.tensor([length for _, length in sizes], dtype=torch.int32, device=dev)
        first = [0]
        for m, _ in sizes:
            first.append(first[-1] + m)
        self.first = first
        self.starts = torch.tensor(first, dtype=torch.int32, device=dev)
        self.rows = first[-1]
        self.cache = Bd.KvCache(self.k, self.v, self.k_scale, self.v_scale)
        self.batch = Bd.KvBatch(self.pages, self.lengths, self.starts)

    def new(self, heads, dtype, rows=None, size=1.0):
        return (torch.randn(self.rows if rows is None else rows, heads, self.dim, generator=self.gen, device=self.dev) * size).to(dtype)

    def places(self, b, first, last):
        p = torch.arange(first, last, device=self.dev)
        return self.pages[b].long()[p // self.page], p % self.page

    def sequence(self, b, t):
        """Values of sequence b's positions in 64 bits and their scales: [kv_heads, positions, dim], [kv_heads, positions]."""
        at, slot = self.places(b, 0, self.sizes[b][1])
        q, s = getattr(self, t)[at, :, slot], getattr(self, t + "_scale")[at, :, slot]
        return q.transpose(0, 1).double(), s.transpose(0, 1).double()

    def attention(self, q, scale=None, window=0, gone=None):
        """(o, tolerance of each of its elements) in 64 bits; gone: positions of the first sequence that are not there.

        Beside the output's own half step, off is: a weight by its rounding to fp16, 2^-11 of it, or 2^-25 of the largest (weight times scale
        of the value) where it is small (a row of zeros counts with the scale 2^-60, scales below 2^-100 as that: such a position may have all of the weight and be the
        largest by it); and by what fp32 does to its exponent: a dot product of `dim` products in any order, each
        addition off by 2^-23 of the sum of the moduli at most (tensor cores cut off), then a product with two rounded factors, an added logarithm and
        the subtraction of the maximum (2^-22 of the largest of the numbers in hand, in log2 units), the exponential, the inverse of the
        scale and the sum of the weights over up to `positions` terms in fp32, each of these to 2^-22 (sum: 2^-24 for each of the terms added one by one)."""
        heads = q.shape[1]
        group, dim = heads // self.kv_heads, self.dim
        scale = dim ** -0.5 if scale is None else scale
        out, tol = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        for b, (n, length) in enumerate(self.sizes):
            if n == 0 or length <= 0:
                continue
            kq, ks = self.sequence(b, "k")
            vq, vs = self.sequence(b, "v")
            K, V = kq * ks[..., None], vq * vs[..., None]
            at = torch.arange(length - n, length, device=q.device)[:, None]
            j = torch.arange(length, device=q.device)
            seen = j <= at
            if window:
                seen &= j > at - window
            if gone is not None and b == 0:
                seen[:, gone] = False
            for h in range(heads):
                c = h // group
                x = q[self.first[b]:self.first[b] + n, h].double()
                s = (x @ K[c].T) * scale
                s = torch.where(seen, s, -math.inf)
                top = s.amax(1, keepdim=True)
                e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
                total = e.sum(1, keepdim=True)
                w = e / torch.where(total > 0, total, 1.0)
                o = w @ V[c]
                moduli = (x.abs() @ K[c].abs().T) * scale * 1.4427
                off = 0.6932 * (torch.where(seen, moduli, 0.0).amax(1, keepdim=True) * dim * 2.0 ** -23 +
                                (torch.where(seen, s, 0.0).abs().amax(1, keepdim=True) * 1.4427 + vs[c].clamp(min=1e-30).log2().abs().max() + 16) * 2.0 ** -22)
                off = off + 4 * 2.0 ** -22 + min(length, 4096) * 2.0 ** -24
                big = (w * torch.where(vs[c] == 0, 2.0 ** -60, vs[c].clamp(min=2.0 ** -100))).amax(1, keepdim=True) * 127
                near = (2.0 ** -11 + 2 * off) * (w @ V[c].abs()) + seen.sum(1, keepdim=True) * 2.0 ** -25 * big
                rows = slice(self.first[b], self.first[b] + n)
                out[rows, h] = o
                tol[rows, h] = HALF_STEP[q.dtype] * o.abs() + near * (1 + 2.0 ** -8) + 2.0 ** -25 * (q.dtype is torch.float16)
        return out, tol
