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
