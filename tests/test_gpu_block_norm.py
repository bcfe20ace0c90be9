"""The norms between two blocks and their gradient against the formulas in 64 bits.

Bounds: a sum of up to 16,384 terms is taken in fp32 by threads (at most 32 terms each), warps and warps of warps, so it is off by less than
50 x 2^-24 = 3e-6 of the sum of its terms' sizes; a root of it by half of that; what is made of them by a few 2^-24 more.  SUM = 1e-5 covers
these together, relative to the sizes of the terms that make an element.  A gradient of a weight adds, for each of a CTA's rows, one term
(at most 100 rows here unless the test says so, 100 x 2^-24 = 6e-6).  Then the output's own rounding."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
SUM = 1e-5
PAIRS = [(BF16, BF16), (F16, F16), (F32, F32), (F32, BF16), (F32, F16)]


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    yield c
    assert c.device_status()[:4] == [0, 0, 0, 0]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def close(got, want, err, dtype=None):
    """err: what the element may be off by before its own rounding."""
    dtype = dtype or got.dtype
    err = err + HALF_STEP[dtype] * (want.abs() + err) + (2.0 ** -25 if dtype is F16 else 1e-38)
    bad = ~((got.double() - want).abs() <= err)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / err)[bad].max()))


def inputs(rows, d, ts, tb, *, post, gates, seed=0, per_gate=0):
    g = gen(rows * 31 + d + seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    t = {"x": (3 * r(rows, d)).to(ts), "y": (r(rows, d) * torch.exp(r(rows, 1))).to(tb), "w_pre": 1 + 0.3 * r(d), "gate": None, "w_post": None,
         "rows_per_gate": 0}
    if post:
        t["w_post"] = 1 + 0.3 * r(d)
    if gates:
        t["gate"], t["rows_per_gate"] = r(gates, d), per_gate or max(1, -(-rows // gates))
    t["dh"], t["dn"] = r(rows, d).to(ts), r(rows, d).to(tb)
    return t


def gate_of(t, rows):
    return None if t["gate"] is None else t["gate"].double()[torch.arange(rows, device=DEV) // t["rows_per_gate"]]


def forward64(t, *, pre=True, post=False, a=1.0, eps=1e-6):
    """(h, n, size of h's terms) by the formulas."""
    x, y = t["x"].double(), t["y"].double()
    u = y / (y.square().mean(1, keepdim=True) + eps).sqrt() if post else y
    if t["w_post"] is not None:
        u = u * t["w_post"].double()
    g = gate_of(t, x.shape[0])
    if g is not None:
        u = u * g
    h = a * x + u
    n = h / (h.square().mean(1, keepdim=True) + eps).sqrt() if pre else h
    if t["w_pre"] is not None:
        n = n * t["w_pre"].double()
    return h, n, (a * x).abs() + u.abs()


def terms(t, **kw):
    return dict(gate=t["gate"], rows_per_gate=t["rows_per_gate"], w_post=t["w_post"], w_pre=t["w_pre"], **kw)


WIDTHS = [(1, 1), (3, 7), (5, 8), (2, 64), (37, 129), (300, 1024), (7, 1030), (160, 4096), (1, 4096), (33, 5121), (200, 8192), (5, 16384), (150, 10001),
          # rows through the ring in shared memory, at the edges of its threads and of their share of a row
          (700, 8), (700, 264), (400, 2056), (330, 4104), (320, 5128), (310, 6152), (300, 8184),
          # cut between the CTAs of a cluster, and rows that start anywhere
          (297, 8200), (300, 11272), (299, 16384), (400, 2055), (320, 5357), (300, 8191), (298, 12001), (600, 33)]


# ---------------------------------------------------------------------------------------------- forward
@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,d", WIDTHS)
@pytest.mark.parametrize("post,gates,a", [(False, 0, 1.0), (True, 0, 0.5), (False, 1, 1.0), (True, 3, -2.0)])
def test_forward(ctx, rows, d, ts, tb, post, gates, a):
    t = inputs(rows, d, ts, tb, post=post, gates=gates)
    h, n = ctx.block_norm(t["x"], t["y"], **terms(t, residual_scale=a))
    assert h.dtype is ts and n.dtype is tb
    rh, rn, size = forward64(t, post=post, a=a)
    close(h, rh, SUM * size)
    r2 = 1 / (rh.square().mean(1, keepdim=True) + 1e-6).sqrt()
    close(n, rn, 2 * SUM * size * r2 * t["w_pre"].double().abs())


@pytest.mark.parametrize("rows,d", [(3, 7), (40, 1024), (300, 4104), (2, 16384), (300, 9001), (310, 12288), (330, 777)])
def test_int8_rows(ctx, rows, d):
    """n rounded to int8 from fp32: a value that close to a border may land on either side of it, so the integers are compared through
    what the norm itself may be off by."""
    t = inputs(rows, d, BF16, BF16, post=True, gates=1)
    h, q, scale = ctx.block_norm_i8(t["x"], t["y"], **terms(t))
    rh, rn, size = forward64(t, post=True)
    close(h, rh, SUM * size)
    top = rn.abs().amax(1, keepdim=True)
    off = 2 * SUM * (size / (rh.square().mean(1, keepdim=True) + 1e-6).sqrt() * t["w_pre"].double().abs())
    worst = off.amax(1, keepdim=True)
    assert ((scale.double()[:, None] - top / 127).abs() <= worst / 127 + 2.0 ** -23 * top / 127).all()
    assert ((q.double() - rn * 127 / top).abs() <= 0.5 + (off + worst) * 127 / top).all()
    assert (q.abs().amax(1) == 127).all()
    # the same bits with the other outputs in one call, and q of n in fp32 is that of the rows' rounding (in fp32 the sums may be
    # taken in another order than in bf16)
    def all_outputs(x, y):
        h2, n2, q2, s2 = torch.empty_like(x), torch.empty_like(y), ctx.new_int8_rows(rows, d), torch.empty(rows, device=DEV)
        Bd.armor_block_norm(ctx.ctx, x, y, h2, n2, q2, s2, **terms(t))
        return h2, n2, q2, s2
    h2, _, q2, s2 = all_outputs(t["x"], t["y"])
    assert torch.equal(h2, h) and torch.equal(q2, q) and torch.equal(s2, scale)
    _, n2, q2, s2 = all_outputs(t["x"].float(), t["y"].float())
    q3, s3 = ctx.quantize_rows(n2)
    assert torch.equal(q2, q3) and torch.equal(s2, s3)


def test_without_a_branch_without_norms_and_in_place(ctx):
    t = inputs(50, 520, BF16, BF16, post=False, gates=0)
    rn = t["x"].double() / (t["x"].double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    h, n = ctx.block_norm(t["x"])
    assert torch.equal(h, t["x"])
    close(n, rn, SUM * rn.abs())
    h, n = ctx.block_norm(t["x"], t["y"], pre=False)
    want = t["x"].double() + t["y"].double()
    assert torch.equal(h, want.to(BF16)) and torch.equal(n, want.to(BF16))
    h, n = ctx.block_norm(t["x"], t["y"], w_pre=t["w_pre"], post=True)           # a norm without a weight
    t["w_post"] = None
    rh, rn, size = forward64(t, post=True)
    close(h, rh, SUM * size)
    x, y = t["x"].clone(), t["y"].clone()
    Bd.armor_block_norm(ctx.ctx, x, y, x, y, None, None, w_pre=t["w_pre"], post=True)
    assert torch.equal(x, h) and torch.equal(y, n)


@pytest.mark.parametrize("off,ld", [(0, 136), (1, 131), (8, 144)])
def test_rows_of_wider_arrays(ctx, off, ld):
    """Strides of their own for every array, and nothing written but the outputs' elements."""
    rows, d = 9, 128
    t = inputs(rows, d, BF16, BF16, post=True, gates=2)
    want = ctx.block_norm(t["x"], t["y"], **terms(t))

    def wide(v, k):
        w = torch.full((rows + 1, ld + 8 * k), 7.0, dtype=BF16, device=DEV)
        if v is not None:
            w[:rows, off:off + d] = v
        return w, w[:rows, off:off + d]
    (_, x), (_, y), (hb, h), (nb, n) = wide(t["x"], 0), wide(t["y"], 1), wide(None, 2), wide(None, 3)
    Bd.armor_block_norm(ctx.ctx, x, y, h, n, None, None, **terms(t))
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    for b, v in ((hb, h), (nb, n)):
        v.fill_(7.0)
        assert (b == 7.0).all()


def test_rows_of_zeros_and_of_extreme_values(ctx):
    d = 256
    x = torch.randn(6, d, generator=gen(1), device=DEV)
    y = torch.randn(6, d, generator=gen(2), device=DEV)
    clean = ctx.block_norm(x, y, post=True)
    x[1], y[1] = 0, 0
    x[2, 5], y[4, 9] = float("nan"), float("inf")
    h, n = ctx.block_norm(x, y, post=True)
    assert (h[1] == 0).all() and (n[1] == 0).all()
    assert torch.isnan(n[2]).all() and torch.isnan(n[4]).all()
    for r in (0, 3, 5):
        assert torch.equal(h[r], clean[0][r]) and torch.equal(n[r], clean[1][r])
    # eps as it is given
    z = torch.full((2, d), 1e-3, device=DEV)
    _, n = ctx.block_norm(z, eps=1e-2)
    want = 1e-3 / (1e-6 + 1e-2) ** 0.5
    assert ((n.double() - want).abs() < 1e-5 * want).all()
    h, n = ctx.block_norm(torch.empty(0, d, device=DEV), torch.empty(0, d, device=DEV))
    assert h.shape == n.shape == (0, d)


# ---------------------------------------------------------------------------------------------- backward
def backward64(t, h, *, post, pre=True, a=1.0, eps=1e-6):
    """({name: gradient}, {name: sizes of the terms}) from h as it is given."""
    rows, d = h.shape
    h, y, dn, dh = h.double(), t["y"].double(), t["dn"].double(), t["dh"].double()
    one = torch.ones(d, dtype=torch.float64, device=DEV)
    w_pre = one if t["w_pre"] is None else t["w_pre"].double()
    w_post = one if t["w_post"] is None else t["w_post"].double()
    g = dn * w_pre
    if pre:
        r2 = 1 / (h.square().mean(1, keepdim=True) + eps).sqrt()
        hn = h * r2
        full = dh + r2 * (g - hn * (g * hn).mean(1, keepdim=True))
        size = dh.abs() + r2 * (g.abs() + hn.abs() * (g * hn).abs().mean(1, keepdim=True))
    else:
        hn, full, size = h, dh + g, dh.abs() + g.abs()
    r1 = 1 / (y.square().mean(1, keepdim=True) + eps).sqrt() if post else 1.0
    yn = y * r1
    e, esize = full, size
    out, sizes = {"dx": a * full, "dw_pre": (dn * hn).sum(0)}, {"dx": abs(a) * size, "dw_pre": (dn * hn).abs().sum(0)}
    gate = gate_of(t, rows)
    if gate is not None:
        at = torch.arange(rows, device=DEV) // t["rows_per_gate"]
        u = yn * w_post
        out["dgate"] = torch.zeros_like(t["gate"], dtype=torch.float64).index_add_(0, at, full * u)
        sizes["dgate"] = torch.zeros_like(out["dgate"]).index_add_(0, at, size * u.abs())
        e, esize = full * gate, size * gate.abs()
    out["dw_post"], sizes["dw_post"] = (e * yn).sum(0), (esize * yn.abs()).sum(0)
    f, fsize = e * w_post, esize * w_post.abs()
    if post:
        out["dy"] = r1 * (f - yn * (f * yn).mean(1, keepdim=True))
        sizes["dy"] = r1 * (fsize + yn.abs() * (fsize * yn.abs()).mean(1, keepdim=True))
    else:
        out["dy"], sizes["dy"] = f, fsize
    return out, sizes


def check_backward(got, want, sizes, times=2):
    for name, v in got.items():
        close(v, want[name].reshape(v.shape), times * SUM * sizes[name].reshape(v.shape))


@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,d", WIDTHS + [(1000, 512)])
@pytest.mark.parametrize("post,gates,a", [(False, 0, 1.0), (True, 0, 0.5), (False, 1, 1.0), (True, 3, -2.0)])
def test_backward(ctx, rows, d, ts, tb, post, gates, a):
    t = inputs(rows, d, ts, tb, post=post, gates=gates)
    got = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t, residual_scale=a))
    assert set(got) == {"dx", "dy", "dw_pre"} | ({"dw_post"} if post else set()) | ({"dgate"} if gates else set())
    want, sizes = backward64(t, t["x"], post=post, a=a)
    check_backward(got, want, sizes)


@pytest.mark.parametrize("rows,gates,per_gate", [(700, 700, 1), (700, 234, 3), (701, 2, 400), (700, 5, 140), (700, 20, 50), (296, 300, 1), (1500, 7, 300), (5, 1, 10)])
def test_gates_of_any_number_of_rows(ctx, rows, gates, per_gate):
    """Gates whose rows lie within one CTA's, span several, end at a CTA's border, or are none (their gradient is zero)."""
    t = inputs(rows, 264, F32, F32, post=True, gates=gates, per_gate=per_gate)
    h, n = ctx.block_norm(t["x"], t["y"], **terms(t))
    rh, rn, size = forward64(t, post=True)
    close(h, rh, SUM * size)
    got = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t))
    want, sizes = backward64(t, t["x"], post=True)
    check_backward(got, want, sizes)
    again = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t))
    assert all(torch.equal(got[k], again[k]) for k in got)


def test_gradient_is_that_of_the_forward_pass(ctx):
    """Central differences of <dh, h> + <dn, n>, by the formulas in 64 bits along a direction for each leaf, against the kernel's gradients.
    The differences are good to about 1e-8 of the terms, the kernel's sums to SUM of the sizes."""
    rows, d = 23, 136
    t = inputs(rows, d, F32, F32, post=True, gates=4)
    h, _ = ctx.block_norm(t["x"], t["y"], **terms(t, residual_scale=0.7))
    got = ctx.block_norm_backward(h, t["y"], t["dh"], t["dn"], **terms(t, residual_scale=0.7))

    def loss(s):
        hh, nn, _ = forward64(s, post=True, a=0.7)
        return float((hh * s["dh"].double()).sum() + (nn * s["dn"].double()).sum())
    for leaf, name in (("x", "dx"), ("y", "dy"), ("w_pre", "dw_pre"), ("w_post", "dw_post"), ("gate", "dgate")):
        v = torch.randn(t[leaf].shape, generator=gen(5), device=DEV, dtype=torch.float64)
        step = 1e-5
        up, down = ({**t, leaf: t[leaf].double() + s * step * v} for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * step)
        along = float((got[name].double() * v).sum())
        assert abs(along - slope) <= 2e-5 * float((got[name].double() * v).abs().sum()) + 1e-6, (name, along, slope)


def test_some_of_the_gradients(ctx):
    """Either incoming gradient may be missing, any outgoing one may be left out, and none changes the others."""
    t = inputs(60, 520, BF16, BF16, post=True, gates=2)
    kw = terms(t)
    full = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **kw)
    zero = torch.zeros_like(t["dh"])
    for dh, dn in ((None, t["dn"]), (t["dh"], None)):
        a = ctx.block_norm_backward(t["x"], t["y"], dh, dn, **kw)
        b = ctx.block_norm_backward(t["x"], t["y"], zero if dh is None else dh, zero if dn is None else dn, **kw)
        assert all(torch.equal(a[k], b[k]) for k in a)
    for name in full:
        out = {k: None for k in full}
        out[name] = torch.empty_like(full[name])
        Bd.armor_block_norm_backward(ctx.ctx, t["x"], t["y"], t["dh"], t["dn"], out["dx"], out["dy"], out["dw_post"], out["dw_pre"],
                                     out["dgate"], **kw)
        assert torch.equal(out[name], full[name]), name
    dx, dy = t["dh"].clone(), t["dn"].clone()
    Bd.armor_block_norm_backward(ctx.ctx, t["x"], t["y"], dx, dy, dx, dy, None, None, None, **kw)
    assert torch.equal(dx, full["dx"]) and torch.equal(dy, full["dy"])
    # without either norm and without weights: the additions alone
    got = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], pre=False, residual_scale=0.5)
    want = t["dh"].double() + t["dn"].double()
    assert torch.equal(got["dx"], (0.5 * want).to(BF16)) and torch.equal(got["dy"], want.to(BF16))
    dx = torch.empty_like(t["dh"])
    Bd.armor_block_norm_backward(ctx.ctx, None, None, t["dh"], None, dx, None, None, None, None, pre=False, residual_scale=2.0)
    assert torch.equal(dx, 2 * t["dh"])


def test_no_rows_give_zero_sums(ctx):
    e = torch.empty(0, 64, device=DEV)
    w, gate = torch.ones(64, device=DEV), torch.ones(3, 64, device=DEV)
    got = ctx.block_norm_backward(e, e, e, e, gate=gate, rows_per_gate=1, w_post=w, w_pre=w)
    assert all((got[k] == 0).all() for k in ("dw_pre", "dw_post", "dgate"))


def test_sums_in_a_small_workspace():
    """Fewer CTAs where the workspace holds fewer sums, and a refusal where it holds none."""
    t = inputs(700, 2000, F32, F32, post=True, gates=2)
    small = Bd.ArmorContext(64, 64, 64, device=DEV, h_mode=Bd.H_DIAG, precision=Bd.PREC_SIMT)
    got = small.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t))
    want, sizes = backward64(t, t["x"], post=True)
    check_backward(got, want, sizes, times=5)                   # 5 CTAs of 140 rows: 140 x 2^-24 more
    tiny = Bd.ArmorContext(4, 4, 4, device=DEV, h_mode=Bd.H_DIAG, precision=Bd.PREC_SIMT)
    with pytest.raises(Bd.ArmorError, match="workspace"):
        tiny.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t))


# ---------------------------------------------------------------------------------------------- as they are used
def test_a_block_of_8_bit_layers():
    """Norm to int8, a linear layer, a factorised layer, norm: each step against the same step in 64 bits on what the one before
    gave, eagerly and replayed from a graph on new inputs."""
    d, hidden = 512, 1024
    g = gen(3)
    up = Bd.ArmorContext(hidden, d, 128, device=DEV)
    down = Bd.ArmorContext(d, hidden, 128, device=DEV)
    wq, ws = up.quantize_rows(torch.randn(hidden, d, generator=g, device=DEV) * 0.05)
    eye = torch.eye(128, device=DEV)
    S = torch.randn(d, hidden // 4, 4, generator=g, device=DEV) * 0.05
    S[:, :, 2:] = 0
    M = torch.full((d, hidden // 4), 3, dtype=torch.uint8, device=DEV)
    packed = down.pack_layer_i8(Bd.LayerState(Wbar=S.view(d, hidden), A=eye.repeat(d // 128, 1, 1), B=eye.repeat(hidden // 128, 1, 1),
                                              S=S.view(d, hidden).contiguous(), M=M))
    w1, w2, w3 = (1 + 0.1 * torch.randn(d, generator=g, device=DEV) for _ in range(3))

    def block(x, y):
        h, q, s = up.block_norm_i8(x, y, w_pre=w1)
        a = up.linear_i8(q, wq, ws, x_scale=s)
        b = down.apply_layer_i8(packed, torch.relu(a))
        h2, n2 = down.block_norm(h, b, w_post=w2, w_pre=w3)
        return h, q, s, a, b, h2, n2

    for n in (1, 77, 300):
        x, y = (torch.randn(n, d, generator=g, device=DEV).to(BF16) for _ in range(2))
        h, q, s, a, b, h2, n2 = block(x, y)
        want = (q.double() @ wq.double().t()) * s.double()[:, None] * ws.double()
        assert ((a.double() - want).abs() <= (HALF_STEP[BF16] + 2.0 ** -21) * want.abs()).all()
        t = {"x": h, "y": b, "w_post": w2, "w_pre": w3, "gate": None}
        rh, rn, size = forward64(t, post=True)
        close(h2, rh, SUM * size)
        held = x.clone(), y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = block(*held)
        x2, y2 = (torch.randn(n, d, generator=g, device=DEV).to(BF16) for _ in range(2))
        for p, r in ((x2, y2), (x, y)):
            held[0].copy_(p)
            held[1].copy_(r)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(out, block(p, r)))


def test_gradients_on_two_streams_and_in_a_graph():
    t = [inputs(500, 1032, BF16, BF16, post=True, gates=2, seed=k) for k in range(2)]
    cs = [Bd.ArmorContext(512, 512, 128, device=DEV, h_mode=Bd.H_DIAG) for _ in range(2)]
    call = lambda c, v: c.block_norm_backward(v["x"], v["y"], v["dh"], v["dn"], **terms(v))  # noqa: E731
    want = [call(cs[0], v) for v in t]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for c, v, s in zip(cs, t, streams):
            with torch.cuda.stream(s):
                got.append(call(c, v))
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        assert all(torch.equal(g[n], want[k % 2][n]) for n in g)
    held = {k: v.clone() if torch.is_tensor(v) else v for k, v in t[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(cs[0], held)
    for k in (1, 0):
        for n in held:
            if torch.is_tensor(held[n]):
                held[n].copy_(t[k][n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[k][n]) for n in out)


def test_refused_calls(ctx):
    x = torch.randn(6, 64, device=DEV)
    w, g = torch.ones(64, device=DEV), torch.ones(4, 64, device=DEV)
    for kw in (dict(y=x.to(BF16), x=x.to(F16)), dict(y=x[:5]), dict(y=x[:, :63]), dict(w_post=w[:63]), dict(w_pre=w.double()), dict(gate=g),
               dict(gate=g, rows_per_gate=1), dict(gate=w, post=True, y=None), dict(pre=False, w_pre=w), dict(post=False, w_post=w), dict(x=x.double()),
               dict(x=x.t()), dict(eps=-1.0)):
        kw = {"x": x, "y": x, **kw}
        with pytest.raises((ValueError, Bd.ArmorError)):
            ctx.block_norm(kw.pop("x"), kw.pop("y"), **kw)
    with pytest.raises(Bd.ArmorError):
        ctx.block_norm_backward(x, x, None, None)
    wide = torch.zeros(2, 16385, device=DEV)
    with pytest.raises(Bd.ArmorError, match="size"):
        ctx.block_norm(wide, wide)
    assert ctx.device_status()[:4] == [0, 0, 0, 0]


@pytest.mark.parametrize("rows,d", [(3, 77), (400, 1032), (320, 9000)])
def test_gradient_without_a_branch(ctx, rows, d):
    """h = residual_scale x, n = h / rms(h) w_pre: dx and dw_pre, and no dy."""
    t = inputs(rows, d, BF16, BF16, post=False, gates=0)
    h, _ = ctx.block_norm(t["x"], w_pre=t["w_pre"], residual_scale=0.5)
    got = ctx.block_norm_backward(h, None, t["dh"], t["dn"], w_pre=t["w_pre"], residual_scale=0.5)
    assert sorted(got) == ["dw_pre", "dx"]
    want, sizes = backward64(t, h, post=False, a=0.5)
    check_backward(got, want, sizes)
