"""Rows of the packed arrays that belong to no sequence of a call, before the first one and behind the last: left as they are, by every call."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.kv_reference import DEV, Case, to_int8

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
SIZES = [(3, 20), (40, 50), (2, 9), (0, 4), (5, 30), (33, 70)]


@pytest.fixture()
def ctx():
    c = Bd.ArmorContext(256, 256, 32, device=DEV)
    yield c
    c.close()


def everything(case):
    return [t.clone() for t in (case.k, case.v, case.k_scale, case.v_scale)]


def part(case, a, b):
    """The batch of the sequences a .. b - 1, with its views of the arrays, and its rows."""
    return Bd.KvBatch(case.pages[a:b], case.lengths[a:b], case.starts[a:b + 1]), slice(case.first[a], case.first[b])


@pytest.mark.parametrize("layout", ["heads", "wide"])
@pytest.mark.parametrize("a,b", [(0, 6), (1, 6), (2, 5), (4, 6), (0, 3), (3, 4)])
@pytest.mark.parametrize("dim,dtype", [(64, BF), (128, torch.float32)])
def test_a_part_of_the_sequences(ctx, a, b, dim, dtype, layout):
    case = Case(SIZES, kv_heads=3, dim=dim, layout=layout, seed=a + 7 * b)
    batch, rows = part(case, a, b)
    k, v = case.new(3, dtype), case.new(3, dtype)
    want = everything(case)
    for s in range(a, b):
        n, length = SIZES[s]
        at, slot = case.places(s, length - n, length)
        for i, x in enumerate((k, v)):
            want[i][at, :, slot], want[i + 2][at, :, slot] = to_int8(x[case.first[s]:case.first[s + 1]])
    ctx.kv_write(case.cache, batch, k, v)
    assert all(torch.equal(x, y) for x, y in zip(everything(case), want))
    out = tuple(torch.full_like(x, 3.0) for x in (k, v))
    ctx.kv_read(case.cache, batch, case.rows, dtype, out=out)
    for x, y in zip((k, v), out):
        q, s = to_int8(x[rows])
        assert torch.equal(y[rows], (q.float() * s[..., None]).to(dtype))
        y[rows] = 3.0
        assert (y == 3.0).all()
    q = case.new(6, BF)
    out = torch.full_like(q, 5.0)
    ctx.kv_attend(case.cache, batch, q, out=out)
    exact, tol = case.attention(q)
    assert ((out.double() - exact).abs() <= tol)[rows].all()
    out[rows] = 5.0
    assert (out == 5.0).all()
    assert ctx.device_status()[11] == 0 and ctx.device_status()[3] == 0


def test_offsets_that_begin_far_in(ctx):
    """More rows before the first sequence than a warp has; and a first sequence that is refused: its own rows are read as zeros."""
    case = Case([(4, 30), (2, 9)], kv_heads=2, dim=64)
    case.starts += 50000
    k = case.new(2, BF, rows=50010)
    before = everything(case)
    ctx.kv_write(case.cache, case.batch, k, k)
    at, slot = case.places(0, 26, 30)
    assert torch.equal(case.v[at, :, slot], to_int8(k[50000:50004])[0]) and ctx.device_status()[11] == 0
    case.lengths[0] = 10 ** 6
    out = tuple(torch.full_like(k, 3.0) for _ in "kv")
    ctx.kv_read(case.cache, case.batch, 50010, out=out)
    for x in out:
        assert (x[:50000] == 3.0).all() and (x[50006:] == 3.0).all() and (x[50000:50004] == 0).all() and (x[50004:50006] != 3.0).any()
    assert ctx.device_status()[11] > 0
    held = torch.zeros_like(before[2], dtype=torch.bool)
    for b, (n, length) in enumerate(case.sizes):
        at, slot = case.places(b, length - n, length)
        held[at, :, slot] = True
    for x, y in zip(everything(case), before):
        same = (x == y) if x.dim() == 3 else (x == y).all(-1)
        assert (same | held).all()


def test_padding_writes_nothing(ctx):
    """The rows of a sequence with fewer positions than rows, and rows behind the last: all four arrays hold what they held but for the rows' own places."""
    case = Case([(5, 2), (1, 20)], kv_heads=2, dim=64)
    want = everything(case)
    k, v = case.new(2, BF, rows=9), case.new(2, BF, rows=9)
    for b, rows in ((0, slice(3, 5)), (1, slice(5, 6))):
        length = case.sizes[b][1]
        at, slot = case.places(b, length - (rows.stop - rows.start), length)
        for i, x in enumerate((k, v)):
            want[i][at, :, slot], want[i + 2][at, :, slot] = to_int8(x[rows])
    ctx.kv_write(case.cache, case.batch, k, v)
    assert all(torch.equal(x, y) for x, y in zip(everything(case), want))
    assert ctx.device_status()[11] == 0
