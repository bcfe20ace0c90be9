"""Rows rounded to int8, the products of such rows (dense and with the 2:4 core) and the layer built from them, against the same
operators in 64 bits.  Integers have to be equal; where nothing but a known rounding stands between the two, so have floats."""
import numpy as np
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    yield c
    assert c.device_status()[:4] == [0, 0, 0, 0]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def quantized(x):
    """(q, scale) by the definition, in 64 bits: 127 x is exact there, and the quotient of two such numbers is further from a half than
    its rounding unless it is one."""
    x = x.double()
    top = x.abs().amax(1, keepdim=True) if x.shape[1] else x.new_zeros(x.shape[0], 1)
    fine = torch.isfinite(top) & (top > 0)
    q = torch.where(fine, torch.round(torch.where(fine, x, 0.0) * 127 / torch.where(fine, top, 1.0)), 0.0)
    scale = torch.where(torch.isfinite(top[:, 0]), top[:, 0] / 127, torch.nan).float()
    return q.to(torch.int8), scale


def same_scales(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


# ---------------------------------------------------------------------------------------------- rows to int8
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,cols", [(1, 1), (3, 7), (5, 8), (2, 127), (300, 129), (1, 4096), (37, 1023), (200, 4104), (9, 8193), (2, 33001), (150, 1032)])
def test_rows_are_rounded_as_defined(ctx, n, cols, dtype):
    x = (torch.randn(n, cols, generator=gen(n + cols), device=DEV) * torch.exp(3 * torch.randn(n, 1, generator=gen(1), device=DEV))).to(dtype)
    q, s = ctx.quantize_rows(x)
    rq, rs = quantized(x)
    assert torch.equal(q, rq)
    assert torch.equal(s, rs)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("off,ld", [(0, 520), (8, 520), (1, 517), (3, 520)])
def test_rows_of_a_wider_array_and_what_lies_behind_them(ctx, dtype, off, ld):
    n, cols = 11, 500
    wide = torch.randn(n + 2, ld, generator=gen(5), device=DEV).to(dtype)
    x = wide[:n, off:off + cols]
    buf = torch.full((n + 2, 512), 77, dtype=torch.int8, device=DEV)
    scale = torch.full((n + 2,), 5.0, device=DEV)
    Bd.armor_quantize_rows(ctx.ctx, x, buf[:n, :cols], scale[:n])
    rq, rs = quantized(x)
    assert torch.equal(buf[:n, :cols], rq) and torch.equal(scale[:n], rs)
    assert (buf[n:] == 77).all() and (scale[n:] == 5.0).all()


def test_ties_and_their_neighbours(ctx):
    """Quotients on a half and one fp32 step to either side of it, at several maxima: those are where a quotient in 32 bits may
    land on the wrong side."""
    rows = []
    for top in (127.0, 1.0, 3.7, 0.0123, 1e-20, 1e25, 254.0, 91.3):
        a = np.float32(top)
        k = np.arange(0, 127, dtype=np.float64) + 0.5
        mid = (k * float(a) / 127.0).astype(np.float32)
        vals = np.concatenate([mid, np.nextafter(mid, np.float32(np.inf)), np.nextafter(mid, np.float32(0)), [a]])
        rows.append(np.concatenate([vals, -vals]))
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DEV)
    q, s = ctx.quantize_rows(x)
    rq, rs = quantized(x)
    assert torch.equal(q, rq) and torch.equal(s, rs)
    assert q.min() == -127 and q.max() == 127


@pytest.mark.parametrize("dtype,bits", [(BF16, 7), (F16, 10)])
def test_every_quotient_of_16_bit_rows(ctx, dtype, bits):
    """Every significand as a row's largest, against every number of ten binades below it, of either sign."""
    m = 2 ** bits
    a = torch.arange(m, 2 * m, device=DEV, dtype=torch.float64)
    below = torch.cat([a * 2.0 ** -s for s in range(10)])
    x = torch.where(below[None] <= a[:, None], below[None], 0.0)
    x = torch.cat([x, -x], 1).to(dtype)
    assert torch.equal(x.double().abs().amax(1), a)
    q, s = ctx.quantize_rows(x)
    rq, rs = quantized(x)
    assert torch.equal(q, rq) and torch.equal(s, rs)
    # the rows one by one through a product of ones, whose sums they are
    wq = torch.ones(1, 256, dtype=torch.int8, device=DEV)
    for r in range(0, m, 7):
        cols = x[r:r + 1, r * 8 % (x.shape[1] - 256):][:, :255]
        row = torch.cat([x[r:r + 1, r:r + 1], cols], 1).contiguous()
        y = ctx.linear_i8(row, wq, torch.ones(1, device=DEV), out_dtype=F32)
        rq, rs = quantized(row)
        assert torch.equal(y, rq.float().sum(1, keepdim=True) * rs)


def test_rows_of_extreme_values(ctx):
    inf, nan = float("inf"), float("nan")
    tiny, big = 2.0 ** -149, 3.4e38
    x = torch.tensor([[0.0, -0.0, 0, 0], [inf, 1, 2, 3], [1, -inf, 2, 3], [nan, 1, 2, 3], [1, 2, 3, nan], [inf, nan, 0, 0],
                      [tiny, -tiny, 0, 0], [5 * tiny, 2 * tiny, -3 * tiny, 0], [big, -big, big / 254, 1.0], [2.0 ** -126, 2.0 ** -133, 0, 1e-40],
                      [1e-30, big, 0, 0]], device=DEV)
    q, s = ctx.quantize_rows(x)
    rq, rs = quantized(x)
    assert torch.equal(q, rq)
    same_scales(s, rs)
    assert torch.isnan(s[1:6]).all() and s[0] == 0
    for dt in (BF16, F16):
        y = torch.tensor([[inf, 1.0], [nan, 1.0], [0.0, 0.0], [2.0 ** -24, -2.0 ** -24]], device=DEV).to(dt)
        q, s = ctx.quantize_rows(y)
        rq, rs = quantized(y)
        assert torch.equal(q, rq)
        same_scales(s, rs)


def test_no_rows(ctx):
    q, s = ctx.quantize_rows(torch.empty(0, 64, device=DEV))
    assert q.shape == (0, 64) and s.shape == (0,)


# ---------------------------------------------------------------------------------------------- the dense product
def int8_rows(n, cols, g, low=-127):
    """Rows on 16-byte boundaries with other rows' values behind them."""
    return torch.randint(low, 128, (n, (cols + 15) // 16 * 16), generator=g, device=DEV, dtype=torch.int8)[:, :cols]


def whole(xq, wq):
    """The integer sums, in 64 bits."""
    return (xq.double() @ wq.double().t()).round()


TOKENS = [1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257, 300, 511, 1000]


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("n_out,n_in", [(1, 1), (3, 16), (100, 17), (128, 128), (129, 130), (255, 4096), (512, 1000), (1000, 2049), (4096, 384)])
def test_sums_are_exact(ctx, n, n_out, n_in):
    """Scales that are powers of two: the output is the integer sum, rounded once."""
    g = gen(n * 7 + n_out + n_in)
    xq, wq = int8_rows(n, n_in, g), int8_rows(n_out, n_in, g, -128)
    xs = torch.exp2(torch.randint(-3, 4, (n,), generator=g, device=DEV).float())
    ws = torch.exp2(torch.randint(-3, 4, (n_out,), generator=g, device=DEV).float())
    want = whole(xq, wq) * xs.double()[:, None] * ws.double()
    y = ctx.linear_i8(xq, wq, ws, x_scale=xs, out_dtype=F32)
    assert torch.equal(y, want.float())


@pytest.mark.parametrize("n", [40, 90, 120, 129, 150, 190, 320, 380, 700, 1024])
@pytest.mark.parametrize("n_out,n_in", [(8192, 2048), (14300, 1000), (4096, 5000), (256, 8200)])
def test_sums_of_every_width_of_tile(ctx, n, n_out, n_in):
    g = gen(n + n_out)
    xq, wq = int8_rows(n, n_in, g), int8_rows(n_out, n_in, g, -128)
    one = torch.ones(max(n, n_out), device=DEV)
    y = ctx.linear_i8(xq, wq, one[:n_out], x_scale=one[:n], out_dtype=F32)
    assert torch.equal(y, whole(xq, wq).float())


def test_sums_of_the_largest_products(ctx):
    """-128 x -128 over the longest contraction, and sums beyond 2^24: exact in int32, rounded once to fp32."""
    n_in = 131071
    xq = torch.full((3, 131072), -128, dtype=torch.int8, device=DEV)[:, :n_in]
    wq = torch.full((130, 131072), -128, dtype=torch.int8, device=DEV)
    wq[1] = 127
    wq = wq[:, :n_in]
    one = torch.ones(130, device=DEV)
    y = ctx.linear_i8(xq, wq, one, x_scale=one[:3], out_dtype=F32)
    assert torch.equal(y, whole(xq, wq).float())
    many = torch.full((300, 131072), -128, dtype=torch.int8, device=DEV)[:, :n_in]
    y = ctx.linear_i8(many, wq, one, x_scale=torch.ones(300, device=DEV), out_dtype=F32)
    assert torch.equal(y, whole(xq[:1], wq).float().expand(300, 130))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,n_out,n_in,bias", [(1, 1024, 1024, True), (5, 77, 333, False), (33, 256, 1040, True), (130, 515, 512, True), (400, 384, 777, False),
                                               (700, 1023, 640, True)])
def test_linear_layer(ctx, n, n_out, n_in, bias, dtype):
    """x of each type, rounded on the way.  Beside the integer sum the output has three roundings to fp32 (sum, product of the scales, their
    product) and with a bias one more, then its own."""
    g = gen(n + n_out)
    x = torch.randn(n, n_in, generator=g, device=DEV).mul_(torch.exp(torch.randn(n_in, generator=g, device=DEV))).to(dtype)
    wq, ws = ctx.quantize_rows(torch.randn(n_out, n_in, generator=g, device=DEV) * 0.02)
    b = torch.randn(n_out, generator=g, device=DEV) if bias else None
    y = ctx.linear_i8(x, wq, ws, bias=b)
    assert y.dtype is dtype
    xq, xs = quantized(x)
    want = whole(xq, wq) * xs.double()[:, None] * ws.double()
    err = 4 * 2.0 ** -24 * want.abs()
    if bias:
        want = want + b.double()
        err = err + 2.0 ** -24 * want.abs()
    err = err + HALF_STEP[dtype] * (want.abs() + err) + (2.0 ** -25 if dtype is F16 else 0.0)
    assert ((y.double() - want).abs() <= err).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("n_out,n_in,off", [(1, 1, 0), (300, 7, 0), (129, 129, 1), (1024, 4096, 0), (2048, 1000, 3), (256, 8192, 0), (20000, 4096, 0), (640, 12289, 0)])
def test_one_token_or_two(ctx, n, n_out, n_in, off, dtype):
    """These are rounded by the product itself, except for the widest rows and pieces; rows that start anywhere."""
    g = gen(n * 3 + n_out + n_in)
    x = (torch.randn(n, n_in + 5, generator=g, device=DEV) * 3).to(dtype)[:, off:off + n_in]
    wq, ws = int8_rows(n_out, n_in, g), torch.exp2(torch.randint(-9, -5, (n_out,), generator=g, device=DEV).float())
    y = ctx.linear_i8(x, wq, ws, out_dtype=F32)
    xq, xs = quantized(x)
    want = whole(xq, wq) * xs.double()[:, None] * ws.double()
    assert ((y.double() - want).abs() <= 3 * 2.0 ** -24 * want.abs()).all()
    if n == 2:
        x = x.clone()
        x[1, n_in // 2] = float("nan")
        z = ctx.linear_i8(x, wq, ws, out_dtype=F32)
        assert torch.isnan(z[1]).all() and torch.equal(z[0], y[0])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n", [3, 90, 300])
@pytest.mark.parametrize("n_out,ldy,off", [(130, 136, 0), (131, 140, 1), (129, 133, 2)])
def test_output_rows_of_a_wider_array(ctx, n, n_out, ldy, off, dtype):
    """Nothing but the output's own elements is written."""
    g = gen(n)
    xq, wq = int8_rows(n, 256, g), int8_rows(n_out, 256, g)
    one = torch.ones(max(n, n_out), device=DEV)
    buf = torch.full((n + 3, ldy), 9.0, dtype=dtype, device=DEV)
    Bd.armor_linear_i8(ctx.ctx, xq, one[:n] / 256, wq, one[:n_out] / 256, None, buf[:n, off:off + n_out])
    want = (whole(xq, wq) / 65536).to(dtype)
    assert torch.equal(buf[:n, off:off + n_out], want)
    buf[:n, off:off + n_out] = 9.0
    assert (buf == 9.0).all()


def test_a_token_that_is_not_finite_stays_alone(ctx):
    x = torch.randn(40, 512, generator=gen(2), device=DEV).to(BF16)
    wq, ws = ctx.quantize_rows(torch.randn(256, 512, generator=gen(3), device=DEV))
    clean = ctx.linear_i8(x, wq, ws)
    x[7, 100], x[20, 3] = float("nan"), float("inf")
    y = ctx.linear_i8(x, wq, ws)
    bad = torch.zeros(40, dtype=torch.bool, device=DEV)
    bad[7] = bad[20] = True
    assert torch.isnan(y[bad]).all()
    assert torch.equal(y[~bad], clean[~bad])


def test_tokens_in_chunks_of_the_workspace():
    """A context whose workspace holds 40 tokens of the call."""
    small = Bd.ArmorContext(128, 128, 128, device=DEV, h_mode=Bd.H_DIAG)
    big = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    x = torch.randn(300, 16000, generator=gen(4), device=DEV).to(BF16)
    wq, ws = big.quantize_rows(torch.randn(200, 16000, generator=gen(5), device=DEV))
    assert torch.equal(small.linear_i8(x, wq, ws), big.linear_i8(x, wq, ws))
    one = torch.ones(1, device=DEV)
    with pytest.raises(Bd.ArmorError, match="workspace"):
        tiny = Bd.ArmorContext(4, 4, 4, device=DEV, h_mode=Bd.H_DIAG, precision=Bd.PREC_SIMT)
        tiny.linear_i8(torch.ones(3, 4096, device=DEV), big.new_int8_rows(1, 4096), one)


def test_no_tokens(ctx):
    wq, ws = ctx.quantize_rows(torch.ones(8, 64, device=DEV))
    assert ctx.linear_i8(torch.empty(0, 64, device=DEV), wq, ws).shape == (0, 8)


def test_weights_written_just_before(ctx):
    """The weight is fetched ahead of the wait for the kernel that rounds the tokens: what wrote it in the same stream has ended by then."""
    x = torch.randn(4, 1024, generator=gen(6), device=DEV).to(BF16)
    for k in range(20):
        w = torch.randn(1024, 1024, generator=gen(100 + k), device=DEV)
        wq, ws = ctx.quantize_rows(w)
        y = ctx.linear_i8(x, wq, ws)
        xq, xs = quantized(x)
        want = whole(xq, quantized(w)[0]) * xs.double()[:, None] * ws.double()
        assert ((y.double() - want).abs() <= (HALF_STEP[BF16] + 2.0 ** -20) * want.abs()).all()


# ---------------------------------------------------------------------------------------------- the layer
def layer(ctx, d_out, d_in, db, seed, exact=False):
    """exact: identity wrappers and a core of whole numbers whose rows have 127 as their largest."""
    g = gen(seed)
    eye = torch.eye(db, device=DEV)
    A, B = (eye.repeat(d // db, 1, 1) if exact else (eye + 0.3 / db ** 0.5 * torch.randn(d // db, db, db, generator=g, device=DEV)).to(BF16).float()
            for d in (d_out, d_in))
    v = torch.randint(-120, 121, (d_out, d_in // 4, 4), generator=g, device=DEV).float() if exact else torch.randn(d_out, d_in // 4, 4, generator=g, device=DEV) * 0.02
    keep = torch.zeros_like(v, dtype=torch.bool).scatter_(2, torch.rand(v.shape, generator=g, device=DEV).topk(2, dim=2).indices, True)
    S = (v * keep).view(d_out, d_in)
    if exact:
        first = keep.view(d_out, d_in).float().argmax(1, keepdim=True)
        S.scatter_(1, first, 127.0)
    M = (keep * torch.tensor([1, 2, 4, 8], device=DEV)).sum(2).to(torch.uint8)
    return Bd.LayerState(Wbar=S, A=A, B=B, S=S, M=M)


SHAPES = [(256, 256, 128), (128, 384, 128), (384, 128, 128), (512, 768, 256), (256, 2048, 256), (1024, 640, 128), (2048, 1024, 128)]


@pytest.mark.parametrize("d_out,d_in,db", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 3, 16, 17, 40, 64, 100, 128, 129, 200, 257, 600, 5000])
def test_core_and_positions_are_exact(d_out, d_in, db, n):
    """Whole numbers throughout: the product with the 2:4 core is an integer, rounded to bf16 on its way to A and not again."""
    c = Bd.ArmorContext(d_out, d_in, db, device=DEV)
    st = layer(c, d_out, d_in, db, d_out + d_in, exact=True)
    x = torch.randint(-120, 121, (n, d_in), generator=gen(n), device=DEV).float()
    x[:, 5] = 127.0
    y = c.apply_layer_i8(c.pack_layer_i8(st), x.to(BF16))
    assert torch.equal(y, (x.double() @ st.S.double().t()).to(BF16))
    assert c.device_status()[:5] == [0, 0, 0, 0, 0]


@pytest.mark.parametrize("n", [40, 90, 120, 250, 500, 1000])
@pytest.mark.parametrize("d_out,d_in", [(8192, 1024), (4096, 2048), (14336, 512)])
def test_core_of_many_rows_is_exact(d_out, d_in, n):
    test_core_and_positions_are_exact(d_out, d_in, 128, n)


@pytest.mark.parametrize("d_out,d_in,db", SHAPES)
@pytest.mark.parametrize("n", [1, 37, 128, 300, 2100, 7000])
@pytest.mark.parametrize("denormalize", [False, True])
def test_layer_against_64_bits(d_out, d_in, db, n, denormalize):
    """Bound, element by element: z1 is an fp32 sum, so where it is within 2^-16 of a step's border its integer may be the other one (counted
    exactly: at most its part of the core's row each); z2 and y are rounded to bf16."""
    c = Bd.ArmorContext(d_out, d_in, db, device=DEV)
    st = layer(c, d_out, d_in, db, 3)
    if denormalize:
        # powers of two: folded into the bf16 wrappers without a rounding
        st.r1 = torch.exp2(torch.randint(-2, 3, (d_in,), generator=gen(8), device=DEV).float())
        st.r2 = torch.exp2(torch.randint(-2, 3, (d_out,), generator=gen(9), device=DEV).float())
    x = (torch.randn(n, d_in, generator=gen(n), device=DEV) * torch.exp(torch.randn(d_in, generator=gen(7), device=DEV))).to(BF16)
    y = c.apply_layer_i8(c.pack_layer_i8(st, denormalize), x).double()
    r1 = st.r1.double() if denormalize else 1.0
    r2 = st.r2.double() if denormalize else 1.0
    z1 = torch.einsum("tjk,jmk->tjm", (x.double() * r1).view(n, -1, db), st.B.double()).reshape(n, d_in)
    top = z1.abs().amax(1, keepdim=True)
    t = z1 * 127 / top
    q = t.round()
    near = ((t - t.floor() - 0.5).abs() < 127 * 2.0 ** -16).double()
    Sq, Ss = quantized(st.S)
    core = Sq.double() * Ss.double()[:, None]
    z2 = (q @ core.t()) * (top / 127)
    moved = (near @ core.abs().t()) * (top / 127) + 2.0 ** -16 * z2.abs()
    z2err = moved + HALF_STEP[BF16] * (z2.abs() + moved)
    want = torch.einsum("tjk,jmk->tjm", z2.view(n, -1, db), st.A.double()).reshape(n, d_out) * r2
    err = torch.einsum("tjk,jmk->tjm", z2err.view(n, -1, db), st.A.double().abs()).reshape(n, d_out) * r2
    err = err * (1 + 2.0 ** -12)
    err = err + HALF_STEP[BF16] * (want.abs() + err)
    assert ((y - want).abs() <= err + 1e-30).all()
    assert float((y - want).norm() / want.norm()) < 4e-3          # two roundings to bf16, each of at most 2^-8 / sqrt(3) on average


def test_groups_that_keep_fewer_or_more_than_two():
    """Fewer: the group's places are filled with zeros.  More: the status word is raised, the first two are taken."""
    d = 256
    c = Bd.ArmorContext(d, d, 128, device=DEV)
    st = layer(c, d, d, 128, 1, exact=True)
    keep = torch.randint(0, 16, (d, d // 4), generator=gen(3), device=DEV)
    count = sum((keep >> k) & 1 for k in range(4))
    st.M = keep.to(torch.uint8)
    vals = torch.randint(-127, 128, (d, d // 4, 4), generator=gen(4), device=DEV).float()
    bits = torch.stack([(keep >> k) & 1 for k in range(4)], 2)
    taken = bits * (bits.cumsum(2) <= 2)
    vals[:, 0], bits[:, 0], taken[:, 0] = 0, 0, 0
    st.M[:, 0], count[:, 0] = 1, 1
    vals[:, 0, 0], taken[:, 0, 0], bits[:, 0, 0] = 127, 1, 1
    st.S = (vals * bits).view(d, d)
    x = torch.randint(-127, 128, (20, d), generator=gen(5), device=DEV).float()
    x[:, 9] = 127
    y = c.apply_layer_i8(c.pack_layer_i8(st), x.to(BF16))
    assert torch.equal(y, (x.double() @ (vals * taken).view(d, d).double().t()).to(BF16))
    # by the words of positions, eight groups each, that hold such a group
    assert c.device_status()[4] == int((count > 2).view(d, -1, 8).any(2).sum())


def test_layer_in_chunks_and_the_rows_behind():
    d_out, d_in = 128, 256
    c = Bd.ArmorContext(d_out, d_in, 128, device=DEV)
    st = layer(c, d_out, d_in, 128, 2, exact=True)
    packed = c.pack_layer_i8(st)
    x = torch.randint(-120, 121, (1024 + 700, d_in), generator=gen(1), device=DEV).float()
    x[:, 0] = 127
    buf = torch.full((x.shape[0] + 4, d_out), 3.0, dtype=BF16, device=DEV)
    Bd.armor_apply_layer_i8(c.ctx, packed, x.to(BF16), buf[:-4])
    assert torch.equal(buf[:-4], (x.double() @ st.S.double().t()).to(BF16)) and (buf[-4:] == 3.0).all()
    assert c.apply_layer_i8(packed, x[:0].to(BF16)).shape == (0, d_out)


def test_layer_with_tokens_that_are_not_finite_or_zero():
    c = Bd.ArmorContext(256, 256, 128, device=DEV)
    packed = c.pack_layer_i8(layer(c, 256, 256, 128, 5))
    for n in (30, 200):
        x = torch.randn(n, 256, generator=gen(n), device=DEV).to(BF16)
        x[3] = 0
        clean = c.apply_layer_i8(packed, x)
        assert (clean[3] == 0).all()
        x[5, 7], x[9, 200] = float("inf"), float("nan")
        y = c.apply_layer_i8(packed, x)
        bad = torch.zeros(n, dtype=torch.bool, device=DEV)
        bad[5] = bad[9] = True
        assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


# ---------------------------------------------------------------------------------------------- as they are used
def test_calls_on_two_streams_and_in_graphs():
    """Two contexts on two streams at once, and each of the calls captured and replayed on new inputs: the bits of plain calls."""
    d_out, d_in = 512, 640
    g = gen(1)
    w = torch.randn(d_out, d_in, generator=g, device=DEV)
    cs = [Bd.ArmorContext(d_out, d_in, 128, device=DEV) for _ in range(2)]
    st = layer(cs[0], d_out, d_in, 128, 4)
    wq, ws = cs[0].quantize_rows(w)
    packed = cs[0].pack_layer_i8(st)
    for n in (3, 150, 400):
        xs = [torch.randn(n, d_in, generator=g, device=DEV).to(BF16) for _ in range(2)]
        want = [(cs[0].linear_i8(x, wq, ws), cs[0].apply_layer_i8(packed, x)) for x in xs]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        got = []
        for _ in range(5):
            for c, x, s in zip(cs, xs, streams):
                with torch.cuda.stream(s):
                    got.append((c.linear_i8(x, wq, ws), c.apply_layer_i8(packed, x)))
        torch.cuda.synchronize()
        for k, pair in enumerate(got):
            assert torch.equal(pair[0], want[k % 2][0]) and torch.equal(pair[1], want[k % 2][1])
        held = xs[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = cs[1].linear_i8(held, wq, ws), cs[1].apply_layer_i8(packed, held)
        for k in (1, 0, 1):
            held.copy_(xs[k])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[k][0]) and torch.equal(out[1], want[k][1])


def test_repeated_calls_give_the_same_bits():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV)
    st = layer(c, 1024, 1024, 128, 6)
    packed = c.pack_layer_i8(st)
    for n in (1, 60, 500):
        x = torch.randn(n, 1024, generator=gen(n), device=DEV).to(BF16)
        first = c.apply_layer_i8(packed, x)
        for _ in range(5):
            assert torch.equal(c.apply_layer_i8(packed, x), first)


def test_launches_are_counted(ctx):
    x = torch.randn(4, 256, device=DEV)
    wq, ws = ctx.quantize_rows(torch.randn(64, 256, device=DEV))
    before = ctx.launch_count()
    ctx.linear_i8(x, wq, ws)
    assert ctx.launch_count() > before


def test_refused_calls(ctx):
    x = torch.randn(4, 64, device=DEV)
    wq, ws = ctx.quantize_rows(torch.randn(8, 64, device=DEV))
    for bad in (dict(x=x.double()), dict(x=x[:, ::2]), dict(x=x[0]), dict(x=x[:, :63]), dict(wq=wq.float()), dict(ws=ws[:7]), dict(bias=ws[:7]),
                dict(x=wq.contiguous()), dict(x_scale=ws), dict(x=x.cpu()), dict(ws=ws.double())):
        args = {"x": x, "wq": wq, "ws": ws, "bias": None, "x_scale": None, **bad}
        with pytest.raises((ValueError, Bd.ArmorError)):
            ctx.linear_i8(args["x"], args["wq"], args["ws"], bias=args["bias"], x_scale=args["x_scale"])
    odd = torch.zeros(8, 70, dtype=torch.int8, device=DEV)[:, :64]
    with pytest.raises(Bd.ArmorError, match="shape"):
        ctx.linear_i8(x, odd, ws)
    with pytest.raises(ValueError):
        Bd.armor_quantize_rows(ctx.ctx, x, odd[:4, :60], ws[:4])
    small = Bd.ArmorContext(64, 64, 64, device=DEV, h_mode=Bd.H_DIAG, precision=Bd.PREC_SIMT)
    with pytest.raises(Bd.ArmorError, match="not supported"):
        small.pack_layer_i8(Bd.LayerState(*[torch.zeros(64, 64, device=DEV)] * 4, M=torch.zeros(64, 16, dtype=torch.uint8, device=DEV)))
    assert ctx.device_status()[:4] == [0, 0, 0, 0]
