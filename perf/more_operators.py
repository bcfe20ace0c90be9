"""Attention over a paged cache of keys and values held as int8 rows with a scale each, and the cache's own two operators: what lies
between the linear layers of a served model's block.

  write   the keys and values of new tokens rounded to int8 rows with a scale each and put in their places in the cache's pages; the pass
          returns them as they are read back
  read    positions of sequences gathered from their pages, as 16- or 32-bit numbers
  attend  a chunk of new tokens of each sequence (one in decoding) against all positions of the sequence up to each token's own

A batch is ``starts`` (rows of the packed arrays that belong to a sequence), ``lengths`` (positions of a sequence, its new tokens among
them: the rows are its last positions) and ``pages`` (its pages in order).  Widths are those of
``paper_2510_05528_b200.inputs.CONFIGS`` in heads of 128 (4096 / 128 query heads, 1024 / 128 key heads, ...) or generic."""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------ the cases
def _case(kind, shape, seqs, chunk, context, *, kv_heads, group=1, dim=128, page=64, dtype="bf16", window=0, name=None):
    """shape: how `seqs` sequences share sizes out: "even" (every chunk `chunk`, context from a quarter of `context` to all of it), "one"
    (the first sequence has the chunk, the others one token each).  chunk 0: whole sequences."""
    c = {"kind": kind, "shape": shape, "seqs": seqs, "chunk": chunk, "context": context, "kv_heads": kv_heads, "group": group, "dim": dim,
         "page": page, "dtype": dtype, "window": window}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decoding step of 64 streams; the chunks of a prompt's step, pages whose size is no power of two; a short fp32 chunk, narrow heads
        _case("write", "even", 64, 1, 4000, kv_heads=8, name="write_64"),
        _case("write", "even", 4, 2047, 6001, kv_heads=8, page=48, name="write_8188"),
        # a short sequence read back whole; a batch of long ones, handed on in 16 bits
        _case("read", "even", 1, 0, 777, kv_heads=8, dtype="f32", name="read_777"),
        _case("read", "even", 16, 0, 12001, kv_heads=8, page=128, name="read_batch"),
        # one stream decoding: latency
        _case("attend", "even", 1, 1, 777, kv_heads=8, group=4, name="attend_1"),
        # a decoding step of 64 streams of any length
        _case("attend", "even", 64, 1, 8000, kv_heads=8, group=4, name="attend_64"),
        # one stream far into a long document
        _case("attend", "even", 1, 1, 131077, kv_heads=8, group=8, page=128, dtype="f16", name="attend_long"),
        # five drafted tokens each for 16 streams
        _case("attend", "even", 16, 5, 4003, kv_heads=8, group=5, page=16, name="attend_drafts"),
        # a chunk of a new prompt beside 40 decoding streams
        _case("attend", "one", 41, 1000, 3001, kv_heads=8, group=4, page=32, name="attend_mixed"),
        # a layer with a sliding window and narrow heads that share no keys
        _case("attend", "even", 4, 1500, 5000, kv_heads=16, dim=64, dtype="f16", window=1024, name="attend_window"),
        # the second chunk of a long prompt, no shared keys; a whole prompt through the widest layer
        _case("attend", "even", 1, 2048, 16385, kv_heads=32, page=64, name="attend_chunk"),
        _case("attend", "even", 1, 8192, 8192, kv_heads=8, group=8, name="attend_prompt"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_once(rng):
    kind = rng.choice(["write", "read", "attend", "attend", "attend", "attend"])
    seqs = _log(rng, 1, 96)
    page = rng.choice([8, 16, 17, 32, 48, 64, 64, 100, 128, 256])
    kv_heads, dim = rng.choice([1, 2, 4, 8, 8, 8, 16, 32]), rng.choice([64, 128, 128])
    group = rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 8, 16])
    if kind != "attend":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        context = _log(rng, 1, 64) if rng.random() < 0.2 else _log(rng, 64, 16384)
        chunk = 0 if kind == "read" and rng.random() < 0.5 else min(context, _log(rng, 1, 8192))
        return _case(kind, "even", seqs, chunk, context, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    window = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
    form = rng.choice(["decode", "decode", "drafts", "mixed", "chunks", "chunks"])
    context = _log(rng, 1, 64) if rng.random() < 0.15 else _log(rng, 64, 131072 if form == "decode" else 32768)
    chunk = {"decode": 1, "drafts": rng.randint(2, 8)}.get(form, _log(rng, 16, 8192))
    return _case("attend", "one" if form == "mixed" else "even", seqs, min(chunk, context), context, kv_heads=kv_heads, group=group, dim=dim,
                 page=page, dtype=dtype, window=window)


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def draw(rng):
    """Another case of the same ranges that costs no more than the largest listed one of its kind, in a cache that is no larger."""
    most, held = {}, max(_held(c) for c in listed())
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        case = _draw_once(rng)
        if _held(case) <= held and _cost(case) <= most[case["kind"]]:
            return case


def _sizes(case):
    """(new tokens, positions) of every sequence: by the case alone."""
    rng = random.Random(",".join(f"{k}={v}" for k, v in sorted(case.items()) if k != "name"))
    out = []
    for b in range(case["seqs"]):
        length = case["context"] if b == 0 else rng.randint(max(1, case["context"] // 4), case["context"])
        new = case["chunk"] or length
        if case["shape"] == "one" and b:
            new = 1
        out.append((min(new, length), length))
    return out


def _held(case):
    pages = sum(-(-length // case["page"]) for _, length in _sizes(case))
    return pages * case["page"] * case["kv_heads"] * (case["dim"] + 4) * 2


# ------------------------------------------------------------------------------------------------ inputs
def _rows_to_int8(x):
    """int8 rows (the last dimension) and their scales: s = max |x| / 127, q = x / s rounded to the nearest, ties to even.  In 64 bits, where
    a quotient that lies next to a border stays on its side."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, torch.round(x * 127.0 / torch.where(top > 0, top, 1.0)), 0.0)
    return q.to(torch.int8), (top[..., 0] / 127.0).float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kv, dim, page, dtype = case["kv_heads"], case["dim"], case["page"], TYPES[case["dtype"]]
    heads = kv * case["group"]
    sizes = _sizes(case)
    st = {"case": case, "sizes": sizes}
    rows = sum(n for n, _ in sizes)
    need = [-(-length // page) for _, length in sizes]
    n_pages = sum(need)
    order = torch.randperm(n_pages, generator=gen, device=DEV).int()
    st["pages"] = torch.zeros(len(sizes), max(need), dtype=torch.int32, device=DEV)
    first = 0
    for b, n in enumerate(need):
        st["pages"][b, :n] = order[first:first + n]
        first += n
    st["lengths"] = torch.tensor([length for _, length in sizes], dtype=torch.int32, device=DEV)
    st["starts"] = torch.tensor([sum(n for n, _ in sizes[:b]) for b in range(len(sizes) + 1)], dtype=torch.int32, device=DEV)
    st["rows"] = rows

    # keys: channels of log-normal spread, two of them wide; values: tokens of log-normal size
    spread = torch.exp(0.4 * torch.randn(kv, 1, dim, generator=gen, device=DEV))
    spread[..., torch.randperm(dim, generator=gen, device=DEV)[:2]] *= 6.0
    cache = {}
    for t in "kv":
        cache[t] = torch.empty(n_pages, kv, page, dim, dtype=torch.int8, device=DEV)
        cache[t + "_scale"] = torch.empty(n_pages, kv, page, device=DEV)
    step = max(1, (1 << 24) // (kv * page * dim))
    for a in range(0, n_pages, step):
        b = min(n_pages, a + step)
        k = torch.randn(b - a, kv, page, dim, generator=gen, device=DEV).mul_(spread)
        v = torch.randn(b - a, kv, page, dim, generator=gen, device=DEV)
        v.mul_(torch.exp(0.5 * torch.randn(b - a, kv, page, 1, generator=gen, device=DEV)))
        for t, x in (("k", k), ("v", v)):
            cache[t][a:b], cache[t + "_scale"][a:b] = _rows_to_int8(x)
    # a sequence's first token draws much of the attention and has little to say
    lean = torch.randn(kv, dim, generator=gen, device=DEV) / spread[:, 0]
    front = st["pages"][:, 0].long()
    sink = 1.5 * lean * spread[:, 0].square()
    cache["k"][front, :, 0], cache["k_scale"][front, :, 0] = _rows_to_int8(sink.expand(len(sizes), kv, dim))
    cache["v_scale"][front, :, 0] *= 0.02
    st.update(cache)

    if case["kind"] != "read":
        # new tokens as a product of all three wrote them: rows of query heads, key heads, value heads
        fused = torch.empty(rows, heads + 2 * kv, dim, dtype=dtype, device=DEV)
        q = 2.0 * torch.randn(rows, kv, case["group"], dim, generator=gen, device=DEV) / spread + 0.5 * lean[:, None]
        fused[:, :heads] = q.reshape(rows, heads, dim).to(dtype)
        fused[:, heads:heads + kv] = torch.randn(rows, kv, dim, generator=gen, device=DEV).mul_(spread[:, 0]).to(dtype)
        fused[:, heads + kv:] = torch.randn(rows, kv, dim, generator=gen, device=DEV).to(dtype)
        st["q"], st["new_k"], st["new_v"] = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
    if own:
        from paper_2510_05528_b200 import binding as Bd
        st["ctx"] = Bd.ArmorContext(4096, 4096, 128, device=DEV, h_mode=Bd.H_DIAG)
        st["cache"] = Bd.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
        st["batch"] = Bd.KvBatch(st["pages"], st["lengths"], st["starts"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _gathered(st, b, length, t):
    """The keys or values of sequence b: [positions, kv_heads, dim]."""
    p = torch.arange(length, device=DEV)
    at, slot = st["pages"][b].long()[p // st["case"]["page"]], p % st["case"]["page"]
    return st[t][at, :, slot].float() * st[t + "_scale"][at, :, slot][..., None]


def run(st):
    case = st["case"]
    kind, dtype = case["kind"], TYPES[case["dtype"]]
    if own:
        ctx, cache, batch = st["ctx"], st["cache"], st["batch"]
        if kind == "attend":
            return ctx.kv_attend(cache, batch, st["q"], window=case["window"])
        if kind == "write":
            ctx.kv_write(cache, batch, st["new_k"], st["new_v"])
        return ctx.kv_read(cache, batch, st["rows"], dtype)

    kv, group, dim = case["kv_heads"], case["group"], case["dim"]
    if kind != "attend":
        t = torch.arange(st["rows"], device=DEV)
        b = torch.searchsorted(st["starts"][1:], t, right=True)
        p = t + (st["lengths"] - st["starts"][1:])[b]
        at, slot = st["pages"][b, p // case["page"]].long(), p % case["page"]
        if kind == "write":
            for t in "kv":
                st[t][at, :, slot], st[t + "_scale"][at, :, slot] = _rows_to_int8(st["new_" + t])
        return tuple((st[t][at, :, slot].float() * st[t + "_scale"][at, :, slot][..., None]).to(dtype) for t in "kv")

    out = torch.empty(st["rows"], kv * group, dim, dtype=dtype, device=DEV)
    row = 0
    for b, (n, length) in enumerate(st["sizes"]):
        k = _gathered(st, b, length, "k").permute(1, 2, 0)                                # [kv_heads, dim, positions]
        v = _gathered(st, b, length, "v").transpose(0, 1)
        step = max(1, (1 << 28) // (length * kv * group))                                   # rows at a time: a gigabyte of weights
        for i in range(0, n, step):
            m = min(step, n - i)
            q = st["q"][row + i:row + i + m].float().view(m, kv, group, dim).permute(1, 0, 2, 3).reshape(kv, m * group, dim)
            s = (q @ k).mul_(1.0 / math.sqrt(dim)).view(kv, m, group, length)
            at = torch.arange(length - n + i, length - n + i + m, device=DEV)[:, None]
            j = torch.arange(length, device=DEV)
            seen = j <= at
            if case["window"]:
                seen &= j > at - case["window"]
            s.masked_fill_(~seen[:, None], float("-inf"))
            w = s.sub_(s.amax(-1, keepdim=True)).exp_()
            o = (w.view(kv, m * group, length) @ v) / w.sum(-1).view(kv, m * group, 1)
            out[row + i:row + i + m] = o.view(kv, m, group, dim).permute(1, 0, 2, 3).reshape(m, kv * group, dim).to(dtype)
        row += n
    return out


# ------------------------------------------------------------------------------------------------ what it takes
def work(case):
    kv, group, dim, size, window = case["kv_heads"], case["group"], case["dim"], SIZE[case["dtype"]], case["window"]
    sizes = _sizes(case)
    rows = sum(n for n, _ in sizes)
    held = 2.0 * kv * (dim + 4)                          # a position in the cache
    table = 4.0 * sum(-(-length // case["page"]) for _, length in sizes) + 8.0 * len(sizes)
    if case["kind"] == "read":
        return {"bytes": rows * (held + 2.0 * kv * dim * size) + table, "flops": 2.0 * rows * kv * dim}
    if case["kind"] == "write":                          # new rows in, the cache, the same rows back
        return {"bytes": rows * (held + 4.0 * kv * dim * size) + table, "flops": 6.0 * rows * kv * dim}
    positions = pairs = 0
    for n, length in sizes:
        w = window or length
        lo = max(0, length - n + 1 - w)                  # the first position that any of the tokens sees
        positions += length - lo
        pairs += sum(min(w, length - i) for i in range(n))
    return {"bytes": positions * held + 2.0 * rows * kv * group * dim * size + table, "flops": 4.0 * pairs * kv * group * dim}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    kv, group, dim, page = case["kv_heads"], case["group"], case["dim"], case["page"]
    sizes = st["sizes"]

    def slots(b, length):
        """Rows of the cache seen as [n_pages * page] of every head."""
        whole = (st["pages"][b].long()[:, None] * page + torch.arange(page, device=DEV)).flatten()
        return whole[:length]

    def flat(t, head):
        return st[t][:, head].reshape(-1, dim), st[t + "_scale"][:, head].reshape(-1)

    if case["kind"] == "write":
        out = []
        for t in ("new_k", "new_v"):
            x = st[t].double()
            width = x.abs().max(dim=2, keepdim=True).values / 127
            out.append((x / width.where(width > 0, torch.ones_like(width))).round() * width)
        return tuple(out)
    if case["kind"] == "read":
        out = []
        for t in "kv":
            of_heads = []
            for h in range(kv):
                values, scales = flat(t, h)
                at = torch.cat([slots(b, length)[length - n:] for b, (n, length) in enumerate(sizes)])
                of_heads.append(values[at].double() * scales[at].double().unsqueeze(1))
            out.append(torch.stack(of_heads, 1))
        return tuple(out)

    out = torch.empty(st["rows"], kv, group, dim, dtype=torch.float64, device=DEV)
    row = 0
    for b, (n, length) in enumerate(sizes):
        at = slots(b, length)
        position = torch.arange(length, device=DEV)
        for h in range(kv):
            values, scales = flat("k", h)
            key = values[at].double() * scales[at].double().unsqueeze(1)
            values, scales = flat("v", h)
            value = values[at].double() * scales[at].double().unsqueeze(1)
            for i in range(0, n, 1024):
                m = min(1024, n - i)
                q = st["q"][row + i:row + i + m, h * group:(h + 1) * group].double()
                mine = position[length - n + i:length - n + i + m].unsqueeze(1)
                hidden = position > mine
                if case["window"]:
                    hidden = hidden | (position <= mine - case["window"])
                for g in range(group):
                    score = torch.where(hidden, -math.inf, torch.einsum("id,jd->ij", q[:, g], key) / dim ** 0.5)
                    out[row + i:row + i + m, h, g] = torch.exp(score - torch.logsumexp(score, 1, keepdim=True)) @ value
        row += n
    return out.view(st["rows"], kv * group, dim)
