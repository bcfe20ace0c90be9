"""The operators that a model of compressed layers is served and tuned with, beside the layers themselves:

  linear     y = x W^T (+ b) on 8-bit integers: the tokens rounded to int8 with a scale each as they come, the weight held
             as int8 with a scale for each of its rows (the linear layers of a model that are not factorised)
  layer      y = A S B x with the kept entries of the 2:4 core as int8, a scale for each row, and the wrapped tokens B x
             rounded to int8 with a scale each (the factorised layers in 8 bits)
  norm       h = a x + gate (.) norm(y) w_post and n = norm(h) w_pre: what lies between a block's last linear layer and the
             first of the next one, norms by the root mean square
  norm_grad  its gradient, with those of the two weights and of the gate

Sizes are those of ``paper_2510_05528_b200.inputs.CONFIGS`` or lie between them."""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases
def _linear(n_out, n_in, tokens, dtype, bias=False, name=None):
    c = {"kind": "linear", "n_out": n_out, "n_in": n_in, "tokens": tokens, "dtype": dtype, "bias": bias}
    return dict(c, name=name) if name else c


def _layer(d_out, d_in, d_block, tokens, name=None):
    c = {"kind": "layer", "d_out": d_out, "d_in": d_in, "d_block": d_block, "tokens": tokens}
    return dict(c, name=name) if name else c


def _norm(kind, rows, d, stream, branch, *, post, gates, scale=1.0, name=None):
    """gates: rows of the gate, each shared by as many consecutive rows (a sequence's); 0: no gate."""
    c = {"kind": kind, "rows": rows, "d": d, "stream": stream, "branch": branch, "post": post, "gates": gates, "scale": scale}
    return dict(c, name=name) if name else c


def listed():
    return [
        # an attention projection in a decoder, one stream: latency, and the reading of the weight
        _linear(4096, 4096, 1, "bf16", name="linear_1"),
        # an up projection, an odd batch of streams
        _linear(14336, 4096, 37, "f16", True, name="linear_37"),
        # a key/value projection over a short prompt whose activations are kept in fp32
        _linear(1024, 5120, 333, "f32", name="linear_kv_333"),
        # the largest up projection over a prompt
        _linear(28672, 8192, 4096, "bf16", name="linear_4096"),
        # factorised layers: one token, an odd batch of streams, a prompt through the largest
        _layer(4096, 4096, 128, 1, name="layer_1"),
        _layer(14336, 4096, 128, 37, name="layer_37"),
        _layer(28672, 8192, 256, 4096, name="layer_4096"),
        # between two blocks: one stream (plain residual addition and the next norm); a ragged prompt with both norms
        # and a gate for the batch
        _norm("norm", 1, 4096, "bf16", "bf16", post=False, gates=0, name="norm_1"),
        _norm("norm", 8195, 8192, "bf16", "bf16", post=True, gates=1, name="norm_8195"),
        # tuning the norms and gates of a compressed model: a batch of short sequences with a gate each; the residual
        # stream in fp32 with a scale; an odd batch in fp16
        _norm("norm_grad", 4096, 4096, "bf16", "bf16", post=True, gates=8, name="grad_4096"),
        _norm("norm_grad", 16384, 5120, "f32", "bf16", post=True, gates=1, scale=0.5, name="grad_f32_stream"),
        _norm("norm_grad", 333, 1024, "f16", "f16", post=False, gates=0, name="grad_333"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _whole(rng, lo, hi):
    return max(lo, min(hi, round(_log(rng, lo, hi))))


def _draw_once(rng):
    kind = rng.choice(["linear", "linear", "layer", "layer", "norm", "norm_grad"])
    if kind == "linear":
        step = rng.choice([1, 8, 16, 128])          # widths off the grid of any tile too
        n_out, n_in = (max(step, round(_log(rng, lo, hi) / step) * step) for lo, hi in ((200, 28672), (200, 14336)))
        return _linear(n_out, n_in, _whole(rng, 1, 8192), rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.5)
    if kind == "layer":
        db = rng.choice([128, 128, 256])
        d_out, d_in = (max(1, round(_log(rng, 512, hi) / db)) * db for hi in (28672, 14336))
        return _layer(d_out, d_in, db, _whole(rng, 1, 8192))
    stream, branch = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f32")])
    rows, d = _whole(rng, 1, 16384), _whole(rng, 64, 16384)
    if rng.random() < 0.7:
        d = max(8, d // 8 * 8)
    gates = rng.choice([0, 1, max(1, min(rows, _whole(rng, 1, 64)))])
    return _norm(kind, rows, d, stream, branch, post=rng.random() < 0.6, gates=gates, scale=rng.choice([1.0, 0.5]))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def draw(rng):
    """Another case of the same ranges that costs no more than the largest listed one of its kind."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most[case["kind"]]:
            return case


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def _activations(gen, tokens, width, dtype):
    """Channels of log-normal standard deviation, one in a thousand an outlier (x 20)."""
    s = torch.exp(0.5 * torch.randn(width, generator=gen, device=DEV))
    s[torch.randperm(width, generator=gen, device=DEV)[: max(1, round(0.001 * width))]] *= 20.0
    return torch.randn(tokens, width, generator=gen, device=DEV).mul_(s).to(dtype)


def _rows_to_int8(x):
    """int8 values and a scale for each row: s = max |x| / 127, q = x / s rounded to the nearest, ties to even.  In 64 bits, where a
    quotient that lies next to a border stays on its side."""
    x = x.double()
    top = x.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(x * 127.0 / torch.where(top > 0, top, 1.0)), 0.0)
    return q.to(torch.int8), (top[:, 0] / 127.0).float()


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "linear":
        n_out, n_in = case["n_out"], case["n_in"]
        st["x"] = _activations(gen, case["tokens"], n_in, TYPES[case["dtype"]])
        # the weight as a program keeps it: int8, rows on 16-byte boundaries
        q = torch.zeros(n_out, (n_in + 15) // 16 * 16, dtype=torch.int8, device=DEV)
        s = torch.empty(n_out, device=DEV)
        for r in range(0, n_out, 4096):
            rows = torch.randn(min(4096, n_out - r), n_in, generator=gen, device=DEV).mul_(0.02)
            q[r:r + 4096, :n_in], s[r:r + 4096] = _rows_to_int8(rows)
        st["wq"], st["ws"] = q[:, :n_in], s
        st["b"] = torch.randn(n_out, generator=gen, device=DEV) if case["bias"] else None
        if own:
            from paper_2510_05528_b200 import binding as Bd
            st["ctx"] = Bd.ArmorContext(4096, 4096, 128, device=DEV, h_mode=Bd.H_DIAG)
    elif kind == "layer":
        d_out, d_in, db = case["d_out"], case["d_in"], case["d_block"]
        eye = torch.eye(db, device=DEV)
        # wrappers near the identity, as a finished layer keeps them: in bf16
        st["A"], st["B"] = ((eye + torch.randn(d // db, db, db, generator=gen, device=DEV).mul_(0.3 / math.sqrt(db))).bfloat16().float()
                            for d in (d_out, d_in))
        g = torch.randn(d_out, d_in // 4, 4, generator=gen, device=DEV).mul_(0.02)
        keep = torch.zeros_like(g, dtype=torch.bool).scatter_(2, g.abs().topk(2, dim=2).indices, True)
        st["M"] = (keep * torch.tensor([1, 2, 4, 8], device=DEV)).sum(2).to(torch.uint8)
        S = g.mul_(keep).view(d_out, d_in)
        st["x"] = _activations(gen, case["tokens"], d_in, torch.bfloat16)
        if own:
            from paper_2510_05528_b200 import binding as Bd
            st["ctx"] = Bd.ArmorContext(d_out, d_in, db, device=DEV)
            st["packed"] = st["ctx"].pack_layer_i8(Bd.LayerState(Wbar=S, A=st["A"], B=st["B"], S=S, M=st["M"]))
        else:
            q, s = torch.empty(d_out, d_in, dtype=torch.int8, device=DEV), torch.empty(d_out, device=DEV)
            for r in range(0, d_out, 4096):
                q[r:r + 4096], s[r:r + 4096] = _rows_to_int8(S[r:r + 4096])
            st["Sq"], st["Ss"] = q, s
    else:
        rows, d = case["rows"], case["d"]
        ts, tb = TYPES[case["stream"]], TYPES[case["branch"]]
        st["x"], st["y"] = _activations(gen, rows, d, ts), _activations(gen, rows, d, tb)
        st["w_pre"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=DEV)
        st["w_post"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=DEV) if case["post"] else None
        st["gate"] = torch.randn(case["gates"], d, generator=gen, device=DEV).mul_(0.5) if case["gates"] else None
        st["per_gate"] = -(-rows // case["gates"]) if case["gates"] else 0
        if kind == "norm_grad":
            # what the forward pass left (h), and the gradients that arrive at its two outputs
            st["h"] = _activations(gen, rows, d, ts)
            st["dh"] = torch.randn(rows, d, generator=gen, device=DEV).to(ts)
            st["dn"] = torch.randn(rows, d, generator=gen, device=DEV).to(tb)
            del st["x"]
        if own:
            from paper_2510_05528_b200 import binding as Bd
            st["ctx"] = Bd.ArmorContext(4096, 4096, 128, device=DEV, h_mode=Bd.H_DIAG)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _gate_rows(st, rows):
    """[rows, d] gate, each of its rows repeated for the rows that share it."""
    return st["gate"].repeat_interleave(st["per_gate"], 0)[:rows]


def _rstd(v):
    return torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        ctx = st["ctx"]
        if kind == "linear":
            return ctx.linear_i8(st["x"], st["wq"], st["ws"], bias=st["b"])
        if kind == "layer":
            return ctx.apply_layer_i8(st["packed"], st["x"])
        terms = dict(gate=st["gate"], rows_per_gate=st["per_gate"], w_post=st["w_post"], w_pre=st["w_pre"],
                     residual_scale=case["scale"], eps=EPS)
        if kind == "norm":
            h, n = ctx.block_norm(st["x"], st["y"], **terms)
            return {"h": h, "n": n}
        return ctx.block_norm_backward(st["h"], st["y"], st["dh"], st["dn"], **terms)

    if kind == "linear":
        q, s = _rows_to_int8(st["x"])
        y = (q.float() @ st["wq"].float().t()) * (s[:, None] * st["ws"])
        return (y if st["b"] is None else y + st["b"]).to(st["x"].dtype)
    if kind == "layer":
        n, db = case["tokens"], case["d_block"]
        z1 = torch.einsum("tjk,jmk->tjm", st["x"].float().view(n, -1, db), st["B"]).reshape(n, -1)
        q, s = _rows_to_int8(z1)
        z2 = (q.float() @ st["Sq"].float().t()) * (s[:, None] * st["Ss"])
        return torch.einsum("tjk,jmk->tjm", z2.view(n, -1, db), st["A"]).reshape(n, -1).bfloat16()
    rows = case["rows"]
    y = st["y"].float()
    r1 = _rstd(y) if case["post"] else None
    yn = y * r1 if case["post"] else y
    u = yn * st["w_post"] if case["post"] else yn
    if kind == "norm":
        x = st["x"].float()
        h = case["scale"] * x + (u * _gate_rows(st, rows) if case["gates"] else u)
        n = h * _rstd(h) * st["w_pre"]
        return {"h": h.to(st["x"].dtype), "n": n.to(st["y"].dtype)}
    h, dn = st["h"].float(), st["dn"].float()
    r2 = _rstd(h)
    hn = h * r2
    g = dn * st["w_pre"]
    dh = st["dh"].float() + r2 * (g - hn * (g * hn).mean(1, keepdim=True))
    out = {"dx": (case["scale"] * dh).to(st["h"].dtype), "dw_pre": (dn * hn).sum(0)}
    e = dh
    if case["gates"]:
        e = dh * _gate_rows(st, rows)
        shared = torch.nn.functional.pad(dh * u, (0, 0, 0, case["gates"] * st["per_gate"] - rows))
        out["dgate"] = shared.view(case["gates"], st["per_gate"], -1).sum(1)
    dy = e
    if case["post"]:
        out["dw_post"] = (e * yn).sum(0)
        f = e * st["w_post"]
        dy = r1 * (f - yn * (f * yn).mean(1, keepdim=True))
    out["dy"] = dy.to(st["y"].dtype)
    return out


# ------------------------------------------------------------------------------------------------ what it takes
def work(case):
    kind = case["kind"]
    if kind == "linear":
        n, o, i, e = case["tokens"], case["n_out"], case["n_in"], SIZE[case["dtype"]]
        return {"bytes": float(o * i + (8 if case["bias"] else 4) * o + e * n * (o + i)), "flops": 2.0 * n * o * i}
    if kind == "layer":
        n, o, i, db = case["tokens"], case["d_out"], case["d_in"], case["d_block"]
        return {"bytes": 0.625 * o * i + 4.0 * o + 2.0 * (o + i) * (db + n), "flops": 2.0 * n * (o * i / 2 + (o + i) * db)}
    n, d = case["rows"], case["d"]
    params = 4.0 * d * (1 + (1 if case["post"] else 0) + case["gates"])
    pair = SIZE[case["stream"]] + SIZE[case["branch"]]
    if kind == "norm":
        return {"bytes": 2.0 * n * d * pair + params, "flops": 12.0 * n * d}
    # reads h and dh, y and dn; writes dx and dy (y is not needed without a norm or a gate of it)
    reads = 2 * pair - (0 if case["post"] or case["gates"] else SIZE[case["branch"]])
    return {"bytes": n * d * float(reads + pair) + 2 * params, "flops": 24.0 * n * d}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _levels(t):
    """The 127 levels to either side that a row of t is rounded to, and their width."""
    width = t.abs().max(dim=1).values.unsqueeze(1) / 127
    return (t / width.where(width > 0, torch.ones_like(width))).round(), width


def _wrapped(t, blocks):
    nb, db, _ = blocks.shape
    return torch.cat([t[:, j * db:(j + 1) * db] @ blocks[j].double().t() for j in range(nb)], 1)


def exact(case, seed):
    kind = case["kind"]
    if kind in ("linear", "layer"):
        o, i = (case["n_out"], case["n_in"]) if kind == "linear" else (case["d_out"], case["d_in"])
        if 2.0 * case["tokens"] * o * i > 1.5e14:
            return None
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if kind == "linear":
        q, width = _levels(st["x"].double())
        y = (q @ st["wq"].double().t()) * width * st["ws"].double()
        return y if st["b"] is None else y + st["b"].double()
    if kind == "layer":
        q, width = _levels(_wrapped(st["x"].double(), st["B"]))
        return _wrapped((q @ st["Sq"].double().t()) * width * st["Ss"].double(), st["A"])
    rows, d = case["rows"], case["d"]

    def rms(t):
        return t / (t.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()

    def leaf(name):
        return None if st[name] is None else st[name].double().requires_grad_()

    y, w_pre, w_post, gate = leaf("y"), leaf("w_pre"), leaf("w_post"), leaf("gate")
    branch = rms(y) * w_post if case["post"] else y
    if case["gates"]:
        branch = branch * gate[torch.arange(rows, device=DEV) // st["per_gate"]]
    if kind == "norm":
        h = case["scale"] * st["x"].double() + branch
        return {"h": h.detach(), "n": (rms(h) * w_pre).detach()}
    # the gradient by automatic differentiation; h enters as what the forward pass left
    h = st["h"].double()
    x = ((h - branch.detach()) / case["scale"]).requires_grad_()
    h = case["scale"] * x + branch
    names = ["dx", "dy", "dw_pre"] + (["dgate"] if case["gates"] else []) + (["dw_post"] if case["post"] else [])
    leaves = {"dx": x, "dy": y, "dw_pre": w_pre, "dgate": gate, "dw_post": w_post}
    got = torch.autograd.grad([h, rms(h) * w_pre], [leaves[n] for n in names], [st["dh"].double(), st["dn"].double()])
    return dict(zip(names, got))
