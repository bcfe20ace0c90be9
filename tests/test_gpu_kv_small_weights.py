"""Attention over many positions of which one has nearly all of the weight: what the others have together is kept."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.kv_heads import attention
from tests.kv_reference import DEV, Case

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
LOST = 2.0 ** -32                            # of the largest contribution: weights are rounded to fp16 with their largest at 2^7 (half of fp16's last place is 2^-25)


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV)
    yield c
    assert c.device_status()[2] == 0 and c.device_status()[11] == 0
    c.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("below", [25.5, 27, 31])
@pytest.mark.parametrize("seqs,new", [(40, 1), (5, 48)])
def test_one_large_weight_and_many_small_ones(ctx, seqs, new, below, dim, dtype):
    """One position has 2^below times the weight of each of 131,071 others and adds nothing to half of the dimensions, whose sum is
    then the others' alone.  The sequences share the pages, and all heads hold the same, so that there are enough units for a CTA to have a whole one."""
    length, heads = 131072 + new - 1, 8 if new == 1 else 32
    one = Case([(new, length)], kv_heads=1, dim=dim, page=64, seed=1, spare=0)
    one.k.zero_()
    one.v.fill_(127)
    one.k_scale.fill_(below * 0.6931472 / 127)
    one.v_scale.fill_(1 / 127)
    page, slot = one.pages[0, 17].long(), 5
    one.k[page, 0, slot, 0] = 127
    one.v[page, 0, slot, dim // 2:] = 0
    q = torch.zeros(new, 1, dim, dtype=dtype, device=DEV)
    q[..., 0] = dim ** 0.5
    want, tol = attention(one, q, lost=LOST)
    assert (want[..., dim // 2:] > 20 * tol[..., dim // 2:]).all() or below == 31
    wide = [t.expand(-1, heads, *t.shape[2:]).contiguous() for t in (one.k, one.v, one.k_scale, one.v_scale)]
    batch = Bd.KvBatch(one.pages.expand(seqs, -1).contiguous(), one.lengths.expand(seqs).contiguous(),
                       torch.arange(seqs + 1, device=DEV, dtype=torch.int32) * new)
    got = ctx.kv_attend(Bd.KvCache(*wide), batch, q.repeat(seqs, heads, 1)).double().view(seqs, new, heads, dim)
    off = (got - want[None]).abs() / tol[None]
    assert (off <= 1).all(), f"{off.max().item():.3g} of the tolerance"


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sizes", [[(1, 700), (1, 40)], [(100, 700), (40, 60)]])
@pytest.mark.parametrize("exponents", [(-20, 20), (-80, -60), (60, 110)])
def test_values_of_all_sizes(ctx, exponents, sizes, dtype):
    """Scales of the values anywhere: the weights' range has room on either side.  (What passes the type's own range is left out: rows whose exact output does.)"""
    case = Case(sizes, kv_heads=2, dim=128, page=32, seed=5)
    gen = case.gen
    case.v_scale.mul_(torch.exp2(torch.randint(*exponents, case.v_scale.shape, generator=gen, device=DEV).float()))
    q = case.new(8, dtype, size=2.0)
    got = ctx.kv_attend(case.cache, case.batch, q)
    want, tol = attention(case, q, lost=LOST)
    least = 2.0 ** -149 if dtype is BF else 0.0          # (bf16's own smallest steps)
    fits = want.abs() <= torch.finfo(dtype).max / 2
    assert fits.any() or (dtype is HF and exponents[0] == 60)
    assert ((got.double() - want).abs() <= tol + least)[fits].all()
