"""The paged cache of int8 keys and values on the GPU: rows in and out."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.kv_reference import DEV, Case, to_int8

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SIZES = [
    [(1, 1)],
    [(1, 17), (0, 5), (3, 3), (1, 64), (0, 0), (40, 100)],
    [(130, 333), (0, 40), (1, 1)],
    [(1, 30 + i) for i in range(70)],
]


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(256, 256, 32, device=DEV)
    yield c
    assert c.device_status()[2] == 0
    c.close()


def everything(case):
    return [t.clone() for t in (case.k, case.v, case.k_scale, case.v_scale)]


@pytest.mark.parametrize("layout", ["heads", "slots", "wide"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,heads,dim,page", [(SIZES[0], 1, 64, 1), (SIZES[1], 3, 128, 16), (SIZES[2], 8, 64, 17), (SIZES[3], 2, 128, 48)])
def test_written_rows_are_the_exact_ones_and_nothing_else_changes(ctx, sizes, heads, dim, page, dtype, layout):
    case = Case(sizes, kv_heads=heads, dim=dim, page=page, layout=layout)
    k, v = case.new(heads, dtype), case.new(heads, dtype, size=30.0)
    want = everything(case)
    for b, (n, length) in enumerate(sizes):
        at, slot = case.places(b, length - n, length)
        rows = slice(case.first[b], case.first[b + 1])
        for i, x in enumerate((k, v)):
            want[i][at, :, slot], want[i + 2][at, :, slot] = to_int8(x[rows])
    ctx.kv_write(case.cache, case.batch, k, v)
    assert all(torch.equal(a, b) for a, b in zip(everything(case), want))
    # and back: what the cache holds, rounded once
    got = ctx.kv_read(case.cache, case.batch, case.rows, dtype)
    for i, x in enumerate(got):
        for b, (n, length) in enumerate(sizes):
            at, slot = case.places(b, length - n, length)
            held = want[i][at, :, slot].float() * want[i + 2][at, :, slot][..., None]
            assert torch.equal(x[case.first[b]:case.first[b + 1]], held.to(dtype))
    assert ctx.device_status()[11] == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_a_wider_array_and_off_a_boundary(ctx, dtype):
    case = Case([(5, 20), (30, 31)], kv_heads=2, dim=64)
    for shift in (0, 1, 8):
        fused = torch.randn(case.rows, 700, generator=case.gen, device=DEV).to(dtype)
        k, v = (fused[:, a + shift:a + shift + 128].view(case.rows, 2, 64) for a in (16, 300))
        ctx.kv_write(case.cache, case.batch, k, v)
        out = torch.full((case.rows, 700), 7.0, dtype=dtype, device=DEV)
        back = tuple(out[:, a + shift:a + shift + 128].view(case.rows, 2, 64) for a in (16, 300))
        ctx.kv_read(case.cache, case.batch, case.rows, dtype, out=back)
        for x, y in ((k, back[0]), (v, back[1])):
            q, s = to_int8(x)
            assert torch.equal(y, (q.float() * s[..., None]).to(dtype))
        out[:, 16 + shift:144 + shift] = 7.0
        out[:, 300 + shift:428 + shift] = 7.0
        assert (out == 7.0).all()


def test_rows_shared_by_heads(ctx):
    """Strides of zero: one row of keys for all heads."""
    case = Case([(3, 9)], kv_heads=4, dim=64)
    k = case.new(1, torch.bfloat16).expand(3, 4, 64)
    ctx.kv_write(case.cache, case.batch, k, k)
    got, _ = ctx.kv_read(case.cache, case.batch, 3)
    q, s = to_int8(k)
    assert torch.equal(got, (q.float() * s[..., None]).bfloat16())


@pytest.mark.parametrize("dtype", TYPES)
def test_special_rows(ctx, dtype):
    """Zeros, rows with NaN or an infinity, the largest and smallest numbers."""
    case = Case([(6, 6)], kv_heads=1, dim=64)
    k = case.new(1, dtype)
    k[0] = 0
    k[1, 0, 5] = float("nan")
    k[2, 0, 63] = -float("inf")
    k[3] = torch.finfo(dtype).max
    k[4] = torch.finfo(dtype).smallest_normal
    ctx.kv_write(case.cache, case.batch, k, k)
    got, _ = ctx.kv_read(case.cache, case.batch, 6, torch.float32)
    assert (got[0] == 0).all() and torch.isnan(got[1:3]).all()
    q, s = to_int8(k[3:])
    assert torch.equal(got[3:], q.float() * s[..., None])


def test_padding_and_rows_behind_the_last_sequence(ctx):
    """More rows than positions: the first stand for positions below zero.  Rows that belong to no sequence are left alone."""
    case = Case([(5, 2), (1, 20)], kv_heads=2, dim=64)
    before = everything(case)
    k = case.new(2, torch.bfloat16, rows=9)
    ctx.kv_write(case.cache, case.batch, k, k)
    at, slot = case.places(0, 0, 2)
    assert torch.equal(case.k[at, :, slot], to_int8(k[3:5])[0])
    at, slot = case.places(1, 19, 20)
    assert torch.equal(case.k[at, :, slot], to_int8(k[5:6])[0])
    assert (torch.stack([a != b for a, b in zip(everything(case)[2:3], before[2:3])]).sum()) <= 3 * 2
    out = tuple(torch.full((9, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.kv_read(case.cache, case.batch, 9, out=out)
    for x in out:
        assert (x[:3] == 0).all() and (x[6:] == 3.0).all() and (x[3:6] != 3.0).any()


def test_pages_out_of_range_are_refused(ctx):
    """(the kernels look at every page, slot and row before they use it)"""
    c = Bd.ArmorContext(256, 256, 32, device=DEV)
    case = Case([(4, 40), (2, 33), (3, 20)], kv_heads=2, dim=64, page=16)
    before = everything(case)
    case.pages[0, 2] = 10 ** 6
    case.pages[1, 2] = -1
    k = case.new(2, torch.bfloat16)
    c.kv_write(case.cache, case.batch, k, k)
    assert c.device_status()[11] > 0 and c.device_status()[3] == 1
    back, _ = c.kv_read(case.cache, case.batch, case.rows)
    assert (back[:4] == 0).all() and (back[5] == 0).all() and (back[6:] != 0).any() and (back[4] != 0).any()
    # positions behind the table, offsets out of order and out of range
    case.lengths[2] = 17 * 16
    case.starts.copy_(torch.tensor([-3, 5, 2, 10 ** 6], dtype=torch.int32))
    c.kv_write(case.cache, case.batch, k, k)
    c.kv_read(case.cache, case.batch, case.rows)
    changed = sum((a != b).any((1, 2, 3)).sum().item() for a, b in zip(everything(case)[:2], before[:2]))
    assert changed <= 2 * 3
    c.close()


def test_captured_calls_follow_what_the_batch_holds(ctx):
    case = Case([(1, 9), (1, 30)], kv_heads=2, dim=128, page=40)       # (lengths grow by three: the table has to hold them)
    k = case.new(2, torch.float16)
    ctx.kv_write(case.cache, case.batch, k, k)
    back = ctx.kv_read(case.cache, case.batch, 2, torch.float16)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.kv_write(case.cache, case.batch, k, k)
        ctx.kv_read(case.cache, case.batch, 2, torch.float16, out=back)
    for step in range(3):
        case.lengths += 1
        k.copy_(case.new(2, torch.float16))
        g.replay()
        q, s = to_int8(k)
        assert torch.equal(back[0], (q.float() * s[..., None]).half())
        for b in range(2):
            at, slot = case.places(b, int(case.lengths[b]) - 1, int(case.lengths[b]))
            assert torch.equal(case.v[at, :, slot], q[b:b + 1])


def test_rows_more_than_2_31_bytes_into_the_cache(ctx):
    page, heads, dim = 256, 8, 128
    n = (2 ** 31) // (page * heads * dim) + 3
    cache = ctx.new_kv_cache(n, page, heads, dim)
    pages = torch.tensor([[n - 1], [0]], dtype=torch.int32, device=DEV)
    batch = Bd.KvBatch(pages, torch.tensor([256, 3], dtype=torch.int32, device=DEV), torch.tensor([0, 2, 3], dtype=torch.int32, device=DEV))
    k = torch.randn(3, heads, dim, device=DEV, dtype=torch.bfloat16)
    ctx.kv_write(cache, batch, k, k)
    q, s = to_int8(k)
    assert torch.equal(cache.v[n - 1, :, 254:].transpose(0, 1), q[:2]) and torch.equal(cache.k[0, :, 2], q[2])
    got, _ = ctx.kv_read(cache, batch, 3)
    assert torch.equal(got, (q.float() * s[..., None]).bfloat16())
