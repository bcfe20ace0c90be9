"""Attention over a paged cache of int8 keys and values against 64 bits."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.kv_reference import DEV, Case

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(2048, 2048, 128, device=DEV)
    yield c
    assert c.device_status()[2] == 0 and c.device_status()[11] == 0
    c.close()


def check(ctx, case, q, **kw):
    got = ctx.kv_attend(case.cache, case.batch, q, **kw)
    kw.pop("max_chunk", None)
    want, tol = case.attention(q, **kw)
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    worst = (off / tol.clamp(min=1e-300)).max().item()
    assert (off <= tol).all(), f"{worst:.3g} of the tolerance"
    return got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,layout", [(16, "heads"), (64, "slots"), (17, "heads"), (1, "wide"), (48, "wide")])
@pytest.mark.parametrize("lengths,kv_heads,group", [
    ([1], 1, 1), ([2, 15, 16, 17, 63, 64, 65], 2, 4), ([1000], 2, 8), ([5, 300], 3, 5), ([129, 1, 640], 1, 16), ([400], 2, 3)])
def test_single_tokens(ctx, lengths, kv_heads, group, page, layout, dim, dtype):
    case = Case([(1, n) for n in lengths], kv_heads=kv_heads, dim=dim, page=page, layout=layout, seed=len(lengths))
    check(ctx, case, case.new(kv_heads * group, dtype, size=3.0))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 9)])
@pytest.mark.parametrize("sizes,kv_heads,group", [
    ([(3, 3)], 1, 1), ([(5, 70), (5, 5), (4, 1000)], 2, 5), ([(100, 100)], 2, 4), ([(257, 300), (1, 90), (0, 40), (33, 33)], 2, 1),
    ([(130, 2000)], 1, 8), ([(1, 64), (65, 129), (2, 2)], 2, 7)])
@pytest.mark.parametrize("window", [0, 1, 50])
def test_chunks(ctx, sizes, kv_heads, group, window, dim, page, dtype):
    case = Case(sizes, kv_heads=kv_heads, dim=dim, page=page, seed=7)
    check(ctx, case, case.new(kv_heads * group, dtype, size=2.0), window=window)
