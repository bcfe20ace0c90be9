"""Arrays whose last rows lie more than 2^31 elements behind the first: the 8-bit products and the norms, all views of one wide array."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    yield c
    assert c.device_status()[:4] == [0, 0, 0, 0]
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_of(base, at, cols, values=None):
    t = base[:, at:at + cols]
    if values is not None:
        t.copy_(values)
    return t


@pytest.mark.parametrize("n,ld", [(2, 2 ** 31 + 16), (37, 2 ** 26 + 16), (2200, 2 ** 20 + 16)])
@pytest.mark.parametrize("off", [0, 3])
def test_rows_to_int8(ctx, n, ld, off):
    x = torch.randn(n, 500, generator=gen(1), device=DEV).to(BF16)
    qx, sx = ctx.quantize_rows(x)
    far = rows_of(torch.empty(n, ld, dtype=BF16, device=DEV), off, 500, x)
    q, s = rows_of(torch.empty(n, ld, dtype=torch.int8, device=DEV), 0, 500), torch.empty(n, device=DEV)
    Bd.armor_quantize_rows(ctx.ctx, far, q, s)
    assert torch.equal(q, qx) and torch.equal(s, sx)


@pytest.mark.parametrize("n,ld", [(2, 2 ** 31 + 16), (37, 2 ** 26 + 16), (300, 2 ** 23 + 16), (2200, 2 ** 20 + 16)])
def test_linear_layer(ctx, n, ld):
    x = torch.randn(n, 400, generator=gen(2), device=DEV).to(BF16)
    w = torch.randn(2100, 400, generator=gen(3), device=DEV)
    wq, ws = ctx.quantize_rows(w)
    want = ctx.linear_i8(x, wq, ws)
    wide = torch.empty(n, ld, dtype=BF16, device=DEV)
    y = rows_of(wide, 4096, 2100)
    far = rows_of(torch.empty(2100, 2 ** 20 + 16, dtype=torch.int8, device=DEV), 0, 400, wq)
    Bd.armor_linear_i8(ctx.ctx, rows_of(wide, 8, 400, x), None, far, ws, None, y)
    assert torch.equal(y, want)
    xq, xs = ctx.quantize_rows(x)
    y.zero_()
    Bd.armor_linear_i8(ctx.ctx, rows_of(torch.empty(n, ld, dtype=torch.int8, device=DEV), 0, 400, xq), xs, far, ws, None, y)
    assert torch.equal(y, want)


def test_packed_layer():
    d, n = 256, 2 ** 23 + 2048
    c = Bd.ArmorContext(d, d, 128, device=DEV, h_mode=Bd.H_DIAG)
    st = c.init(torch.randn(d, d, generator=gen(4), device=DEV), torch.eye(d, device=DEV))
    packed = c.pack_layer_i8(st)
    x = torch.randn(2048, d, generator=gen(5), device=DEV).to(BF16)
    want = c.apply_layer_i8(packed, x)
    far = torch.zeros(n, d, dtype=BF16, device=DEV)
    far[-2048:] = x
    assert torch.equal(c.apply_layer_i8(packed, far)[-2048:], want)
    assert c.device_status()[:4] == [0, 0, 0, 0]


@pytest.mark.parametrize("rows,ld", [(2, 2 ** 31 + 16), (37, 2 ** 26 + 16), (2200, 2 ** 20 + 16)])
@pytest.mark.parametrize("d,off", [(520, 0), (517, 3), (9000, 0)])
def test_norms(ctx, rows, ld, d, off):
    """The same bits as of rows that lie side by side with the same alignment."""
    g = gen(6)
    wide, near = torch.empty(rows, ld, dtype=BF16, device=DEV), torch.empty(rows, 8 * 9216, dtype=BF16, device=DEV)
    terms = dict(gate=torch.randn(2, d, generator=g, device=DEV), rows_per_gate=(rows + 1) // 2, w_post=torch.randn(d, generator=g, device=DEV),
                 w_pre=torch.randn(d, generator=g, device=DEV))
    values = [torch.randn(rows, d, generator=g, device=DEV) for _ in range(4)]
    made = []
    for base in (near, wide):
        x, y, dh, dn = (rows_of(base, 9216 * k + off, d, v) for k, v in enumerate(values))
        h, n, dx, dy = (rows_of(base, 9216 * k + off, d) for k in range(4, 8))
        q, s = ctx.new_int8_rows(rows, d), torch.empty(rows, device=DEV)
        dw = [torch.empty(d, device=DEV), torch.empty(d, device=DEV), torch.empty(2, d, device=DEV)]
        Bd.armor_block_norm(ctx.ctx, x, y, h, n, q, s, **terms)
        Bd.armor_block_norm_backward(ctx.ctx, h, y, dh, dn, dx, dy, *dw, **terms)
        made.append([t.clone() for t in (h, n, q, s, dx, dy, *dw)])
    for a, b in zip(*made):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b)


def test_arrays_in_host_memory_are_refused(ctx):
    x = torch.zeros(4, 32, device=DEV)
    o = torch.empty_like(x)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm(ctx.ctx, x.cpu(), None, o, o, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm(ctx.ctx, x, x.cpu(), o, o, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm(ctx.ctx, x.cpu(), x.cpu(), o, o, None, None, w_pre=torch.ones(32))
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm_backward(ctx.ctx, x.cpu(), x.cpu(), x.cpu(), x.cpu(), o, o, None, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        ctx.block_norm(x, x, w_pre=torch.ones(32))
    with pytest.raises(ValueError, match="CUDA"):
        ctx.linear_i8(x, torch.zeros(32, 32, dtype=torch.int8), torch.ones(32, device=DEV))
    wq, ws = ctx.quantize_rows(x)
    with pytest.raises(ValueError, match="CUDA"):
        ctx.linear_i8(x, wq, ws.cpu())
