"""The attention's tile kernel where a CTA takes many units and many blocks, against 64 bits."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.kv_heads import attention
from tests.kv_line import most, shares
from tests.kv_reference import DEV, Case

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV)
    yield c
    assert c.device_status()[2] == 0 and c.device_status()[11] == 0
    c.close()


def sms():
    return torch.cuda.get_device_properties(DEV).multi_processor_count


def check(ctx, case, q, **kw):
    got = ctx.kv_attend(case.cache, case.batch, q, **kw)
    assert ctx.device_status()[2] == 0
    want, tol = attention(case, q, window=kw.get("window", 0))
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert (off <= tol).all(), f"{(off / tol.clamp(min=1e-300)).max().item():.3g} of the tolerance"
    return got


# ---- prompts of a block each, with sequences that the kernel steps over between them
GAPS = [(22, 38), (60, 15), (30, 45), (75,)]


def test_heads_at_once_are_the_heads_one_by_one():
    case = Case([(5, 70), (0, 9), (4, 2), (300, 400)], kv_heads=2, dim=64, page=16, seed=1)
    case.sizes[2] = (2, 2)                       # (its first two rows are padding)
    case.first = [0, 5, 7, 9]
    q = case.new(6, BF, size=2.0)
    for window in (0, 50):
        for a, b in zip(attention(case, q, window=window), case.attention(q, window=window)):
            assert ((a - b).abs() <= 1e-12 * (1 + b.abs())).all()


@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("gaps", GAPS)
def test_short_prompts_around_many_others(ctx, gaps, empty):
    """Prompts of 16 tokens in a table of 1,024 slots; the other slots decode, or are empty."""
    other = 1024 - sum(gaps)
    each = -(-other // len(gaps))
    sizes = []
    for n in gaps:
        sizes += [(16, 16)] * n
        sizes += [(0, 0) if empty else (1, 1 + i % 40) for i in range(min(each, other))]
        other -= min(each, other)
    sizes += [(16, 16)] * (1024 - len(sizes))
    units = [b for s in shares(sizes, 8, 4, n_ctas=sms()) for b, _ in s]
    assert set(units) == {1} and most(sizes, 8, 4, n_ctas=sms())[0] >= 4
    case = Case(sizes, kv_heads=8, dim=64, page=16, seed=len(gaps))
    for dtype in (BF, HF):
        check(ctx, case, case.new(32, dtype, size=2.0))


def test_prompts_far_apart(ctx):
    """One prompt at a time with some hundred others in front of it: each CTA's few units lie far apart."""
    sizes = ([(1, 3)] * 120 + [(60, 60)] * 9) * 7
    case = Case(sizes, kv_heads=16, dim=64, page=16, seed=4)
    check(ctx, case, case.new(16, BF, size=2.0))
    check(ctx, case, case.new(32, HF, size=2.0))


# ---- many units, many blocks
def mixed(n):
    """Units of one block and of several, tiles of a half and of both, one behind the other."""
    return [((33, 33), (64, 64), (65, 300), (40, 41), (128, 200), (129, 129), (300, 300), (257, 500), (34, 64))[i % 9] for i in range(n)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,page,layout", [(64, 16, "heads"), (128, 17, "slots"), (128, 64, "heads")])
@pytest.mark.parametrize("sizes,kv_heads,group,window,least", [
    ([(9 + i % 56, 9 + i % 56) for i in range(120)], 8, 4, 0, (6, 6)),           # one block each
    (mixed(108), 8, 1, 0, (6, 17)),
    (mixed(54), 4, 5, 0, (6, 17)),
    ([(1400, 2500), (1200, 1200), (1800, 2200)], 16, 2, 256, (6, 17)),               # a window
    (mixed(72), 8, 2, 70, (6, 17)),
])
def test_many_units_a_cta(ctx, sizes, kv_heads, group, window, least, dim, page, layout, dtype):
    got = most(sizes, kv_heads, group, window=window, n_ctas=sms())
    assert got[0] >= least[0] and got[1] >= least[1], got
    case = Case(sizes, kv_heads=kv_heads, dim=dim, page=page, layout=layout, seed=2)
    check(ctx, case, case.new(kv_heads * group, dtype, size=2.0), window=window)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sizes,kv_heads,group,least", [
    ([(1700, 1700)], 8, 8, (6, 40)),                      # a whole prompt
    ([(300, 30000), (40, 60000)], 4, 4, (2, 90)),         # long pieces of cut units
    ([(256, 12000)] * 5, 32, 1, (2, 150)),
])
def test_many_blocks_a_cta(ctx, sizes, kv_heads, group, least, dtype):
    got = most(sizes, kv_heads, group, n_ctas=sms())
    assert got[0] >= least[0] and got[1] >= least[1], got
    case = Case(sizes, kv_heads=kv_heads, dim=128, page=64, seed=3)
    check(ctx, case, case.new(kv_heads * group, dtype, size=2.0))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_units_where_there_is_no_room_for_parts(dim, dtype):
    sizes = mixed(90)
    assert most(sizes, 8, 1, n_ctas=sms(), whole=True)[0] >= 5
    small = Bd.ArmorContext(64, 64, 32, device=DEV, h_mode=Bd.H_DIAG)
    case = Case(sizes, kv_heads=8, dim=dim, page=16, seed=6)
    check(small, case, case.new(8, dtype, size=2.0))
    small.close()


@pytest.mark.parametrize("sizes,kv_heads,group", [(mixed(108), 8, 1), ([(16, 16)] * 100, 8, 4), ([(1700, 1700)], 8, 8)])
def test_runs_give_the_same_bits(ctx, sizes, kv_heads, group):
    case = Case(sizes, kv_heads=kv_heads, dim=128, page=32, seed=8)
    for dtype in (BF, HF):
        q = case.new(kv_heads * group, dtype, size=2.0)
        first = ctx.kv_attend(case.cache, case.batch, q)
        for _ in range(10):
            assert torch.equal(ctx.kv_attend(case.cache, case.batch, q), first)
