"""The norms and their gradient over rows of wider arrays whose width is no multiple of a vector's elements: rows on 16-byte boundaries,
lengths that end inside one.  Bounds as in test_gpu_block_norm.py.  What lies behind an input's row, a weight or a gate is NaN, which reaches every
element of a row whose sums take it in; what lies behind an output is held to stay as it was."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.test_gpu_block_norm import PAIRS, SUM, backward64, check_backward, close, forward64, inputs, terms

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 7.0
# one chunk of a thread's share, two, three; as many as the forward ring takes; the gradient beyond its ring
WIDTHS = [9, 1001, 1002, 1004, 4100, 5357, 8191, 11001]


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    yield c
    assert c.device_status()[:4] == [0, 0, 0, 0]


def wide(v, fill):
    """(array, view of v's shape in it): rows 16 bytes apart at least, on 16-byte boundaries, a row more than v has."""
    rows, d = v.shape
    buf = torch.full((rows + 1, d // 8 * 8 + 8), fill, dtype=v.dtype, device=DEV)
    buf[:rows, :d] = v
    return buf, buf[:rows, :d]


def behind(buf, view):
    """Everything of buf but the view."""
    rest = torch.ones(buf.shape, dtype=torch.bool, device=DEV)
    rest[:view.shape[0], :view.shape[1]] = False
    return buf[rest]


def ending(v):
    """A vector of v's elements with NaN behind it."""
    buf = torch.full((v.numel() + 32,), float("nan"), device=DEV)
    buf[:v.numel()] = v
    return buf[:v.numel()]


def padded(rows, d, ts, tb, gates):
    t = inputs(rows, d, ts, tb, post=True, gates=gates)
    p = {k: wide(t[k], float("nan"))[1] for k in ("x", "y", "dh", "dn")}
    p["gate"] = None if t["gate"] is None else wide(t["gate"], float("nan"))[1]
    p["w_pre"], p["w_post"], p["rows_per_gate"] = ending(t["w_pre"]), ending(t["w_post"]), t["rows_per_gate"]
    return t, p


@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,gates", [(9, 2), (400, 0), (700, 3)])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(ctx, rows, gates, d, ts, tb):
    t, p = padded(rows, d, ts, tb, gates)
    (hb, h), (nb, n) = (wide(torch.full((rows, d), KEPT, dtype=dt, device=DEV), KEPT) for dt in (ts, tb))
    q, scale = ctx.new_int8_rows(rows, d), torch.full((rows + 1,), KEPT, device=DEV)
    Bd.armor_block_norm(ctx.ctx, p["x"], p["y"], h, n, q, scale[:rows], **terms(p))
    assert (behind(hb, h) == KEPT).all() and (behind(nb, n) == KEPT).all() and scale[rows] == KEPT
    rh, rn, size = forward64(t, post=True)
    close(h, rh, SUM * size)
    off = 2 * SUM * size / (rh.square().mean(1, keepdim=True) + 1e-6).sqrt() * t["w_pre"].double().abs()
    close(n, rn, off)
    # int8: within a half step of what the norm may be off by, as in test_gpu_block_norm.test_int8_rows
    top, worst = rn.abs().amax(1, keepdim=True), off.amax(1, keepdim=True)
    assert ((scale[:rows].double()[:, None] - top / 127).abs() <= worst / 127 + 2.0 ** -23 * top / 127).all()
    assert ((q.double() - rn * 127 / top).abs() <= 0.5 + (off + worst) * 127 / top).all()


@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,gates", [(9, 2), (400, 0), (700, 3)])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward(ctx, rows, gates, d, ts, tb):
    t, p = padded(rows, d, ts, tb, gates)
    (xb, dx), (yb, dy) = (wide(torch.full((rows, d), KEPT, dtype=dt, device=DEV), KEPT) for dt in (ts, tb))
    sums = {k: torch.full((n * d + 32,), KEPT, device=DEV) for k, n in (("dw_post", 1), ("dw_pre", 1), ("dgate", gates)) if n}
    got = {k: v[:-32] for k, v in sums.items()}
    Bd.armor_block_norm_backward(ctx.ctx, p["x"], p["y"], p["dh"], p["dn"], dx, dy, got["dw_post"], got["dw_pre"], got.get("dgate"), **terms(p))
    assert (behind(xb, dx) == KEPT).all() and (behind(yb, dy) == KEPT).all()
    assert all((v[-32:] == KEPT).all() for v in sums.values())
    want, sizes = backward64(t, t["x"], post=True)
    check_backward({"dx": dx, "dy": dy, **got}, want, sizes)


@pytest.mark.parametrize("d", [1001, 1004, 5357])
def test_one_array_padded_and_arrays_left_out(ctx, d):
    """The stream alone, as a view of a wider array, and only its int8 rows or only its gradient asked for."""
    rows = 500
    t, p = padded(rows, d, torch.bfloat16, torch.bfloat16, 0)
    q, scale = ctx.new_int8_rows(rows, d), torch.empty(rows, device=DEV)
    Bd.armor_block_norm(ctx.ctx, p["x"], None, None, None, q, scale, w_pre=p["w_pre"])
    qc, sc = ctx.block_norm_i8(t["x"].contiguous(), w_pre=t["w_pre"])[1:]
    assert torch.equal(q, qc) and torch.equal(scale, sc)
    xb, dx = wide(torch.full((rows, d), KEPT, dtype=torch.bfloat16, device=DEV), KEPT)
    Bd.armor_block_norm_backward(ctx.ctx, p["x"], None, None, p["dn"], dx, None, None, None, None, w_pre=p["w_pre"])
    assert torch.equal(dx, ctx.block_norm_backward(t["x"], None, torch.zeros_like(t["x"]), t["dn"], w_pre=t["w_pre"])["dx"])
    assert (behind(xb, dx) == KEPT).all()


@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,d", [(700, 1), (701, 2), (2000, 3), (20000, 5)])
def test_rows_shorter_than_a_vector(ctx, rows, d, ts, tb):
    """Many rows of a few elements, one behind the other: most start and end inside a vector that holds neighbours too."""
    t = inputs(rows, d, ts, tb, post=True, gates=2)
    h, q, scale = ctx.block_norm_i8(t["x"], t["y"], **terms(t))
    n = ctx.block_norm(t["x"], t["y"], **terms(t))[1]
    rh, rn, size = forward64(t, post=True)
    close(h, rh, SUM * size)
    off = 2 * SUM * size / (rh.square().mean(1, keepdim=True) + 1e-6).sqrt() * t["w_pre"].double().abs()
    close(n, rn, off)
    top, worst = rn.abs().amax(1, keepdim=True), off.amax(1, keepdim=True)
    assert ((q.double() - rn * 127 / top).abs() <= 0.5 + (off + worst) * 127 / top).all()
    got = ctx.block_norm_backward(t["x"], t["y"], t["dh"], t["dn"], **terms(t))
    want, sizes = backward64(t, t["x"], post=True)
    check_backward(got, want, sizes)
