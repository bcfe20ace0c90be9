"""The attention over the paged cache in 64 bits, all heads of a sequence at once: for batches of many sequences."""
import torch

from tests.kv_reference import HALF_STEP


def attention(case, q, window=0, lost=2.0 ** -25):
    """(o, tolerance) as Case.attention has them; lost: what a weight's rounding to fp16 may be off by where it is small, of the row's largest."""
    out, tol = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in "ot")
    kv, dim = case.kv_heads, case.dim
    group, scale = q.shape[1] // kv, dim ** -0.5
    for b, (n, length) in enumerate(case.sizes):
        if n == 0 or length <= 0:
            continue
        (kq, ks), (vq, vs) = case.sequence(b, "k"), case.sequence(b, "v")
        K, V, vs = kq * ks[..., None], vq * vs[..., None], vs[:, None]
        at = torch.arange(length - n, length, device=q.device).repeat_interleave(group)[:, None]
        j = torch.arange(length, device=q.device)
        seen = j <= at
        if window:
            seen &= j > at - window
        rows = slice(case.first[b], case.first[b] + n)
        x = q[rows].double().view(n, kv, group, dim).transpose(0, 1).reshape(kv, n * group, dim)
        s = (x @ K.transpose(1, 2)) * scale
        moduli = torch.where(seen, (x.abs() @ K.abs().transpose(1, 2)) * scale * 1.4427, 0.0).amax(-1, keepdim=True)
        most = torch.where(seen, s, 0.0).abs().amax(-1, keepdim=True) * 1.4427
        s = torch.where(seen, s, -torch.inf)
        top = s.amax(-1, keepdim=True)
        w = torch.exp(s - torch.where(top == -torch.inf, 0.0, top))
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
        o = w @ V
        off = 0.6932 * (moduli * dim * 2.0 ** -23 + (most + vs.clamp(min=1e-30).log2().abs().amax(-1, keepdim=True) + 16) * 2.0 ** -22)
        off = off + 4 * 2.0 ** -22 + min(length, 4096) * 2.0 ** -24
        big = (w * torch.where(vs == 0, 2.0 ** -60, vs.clamp(min=2.0 ** -100))).amax(-1, keepdim=True) * 127
        near = (2.0 ** -11 + 2 * off) * (w @ V.abs()) + seen.sum(-1, keepdim=True) * lost * big
        near = HALF_STEP[q.dtype] * o.abs() + near * (1 + 2.0 ** -8) + 2.0 ** -25 * (q.dtype is torch.float16)
        for to, t in ((out, o), (tol, near)):
            to[rows] = t.view(kv, n, group, dim).transpose(0, 1).reshape(n, kv * group, dim)
    return out, tol
