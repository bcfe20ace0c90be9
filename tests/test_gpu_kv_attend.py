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
    kw.pop("out", None)
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


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sizes,kv_heads,group,dim,page,layout", [
    # few rows and many in one batch: both kernels
    ([(1, 700), (300, 301), (0, 0), (4, 4), (1, 1), (64, 2000), (2, 5), (17, 17)], 2, 4, 128, 16, "heads"),
    ([(1, 700), (300, 301), (3, 30), (1, 1)], 1, 5, 64, 24, "slots"),
    # more heads to a key head than one kernel takes rows
    ([(1, 333), (1, 64), (1, 2)], 1, 32, 128, 32, "heads"),
    ([(3, 333)], 2, 33, 64, 16, "wide"),
    # parts of units in many CTAs, few rows and many
    ([(1, 20000)], 1, 8, 128, 64, "heads"), ([(2, 30001)], 1, 7, 64, 16, "slots"), ([(40, 20000)], 1, 1, 128, 64, "heads"), ([(33, 12345)], 2, 4, 64, 48, "heads"),
    # tiles of one row, of a half's rows, one more and one fewer
    ([(127, 127), (128, 128), (129, 129), (255, 255), (256, 256), (257, 257)], 1, 1, 128, 64, "heads"),
    ([(63, 64), (64, 64), (65, 64)], 1, 4, 64, 64, "heads")])
def test_mixtures_and_cuts(ctx, sizes, kv_heads, group, dim, page, layout, dtype):
    case = Case(sizes, kv_heads=kv_heads, dim=dim, page=page, layout=layout, seed=3)
    check(ctx, case, case.new(kv_heads * group, dtype, size=2.0))


@pytest.mark.parametrize("max_chunk", [0, 1, 2, 50, 5000])
def test_the_hint_changes_no_meaning(ctx, max_chunk):
    for sizes in ([(1, 90), (20, 70), (300, 400)], [(1, 900)], [(40, 40)]):
        case = Case(sizes, kv_heads=2, dim=128, page=16, seed=5)
        check(ctx, case, case.new(8, BF, size=2.0), max_chunk=max_chunk)


def test_more_sequences_than_a_launch_takes(ctx):
    sizes = [(1, 1 + i % 50) for i in range(2100)]
    sizes[1500] = (70, 90)
    case = Case(sizes, kv_heads=1, dim=64, page=16, seed=2)
    check(ctx, case, case.new(4, BF))


@pytest.mark.parametrize("scale", [0.0, 0.01, 1.0])
@pytest.mark.parametrize("sizes", [[(1, 300), (5, 9)], [(200, 300)]])
def test_scales(ctx, sizes, scale):
    case = Case(sizes, kv_heads=2, dim=64, page=16, seed=9)
    check(ctx, case, case.new(4, HF), scale=scale)


@pytest.mark.parametrize("sizes", [[(1, 500), (1, 3)], [(150, 500)]])
def test_sharp_rows_and_values_of_all_sizes(ctx, sizes):
    """Scores of hundreds, values over twelve decades (one position in five a hundred times larger), rows of zeros (their scale is 0)."""
    case = Case(sizes, kv_heads=2, dim=128, page=32, seed=11)
    gen = case.gen
    case.v_scale.mul_(torch.exp2(torch.randint(-20, 20, case.v_scale.shape, generator=gen, device=DEV).float()))
    case.k_scale.mul_(4.0)
    for t in "kv":
        zero = torch.rand(case.v_scale.shape, generator=gen, device=DEV) < 0.1
        getattr(case, t).masked_fill_(zero[..., None], 0)
        getattr(case, t + "_scale").masked_fill_(zero, 0.0)
    check(ctx, case, case.new(8, BF, size=4.0))


@pytest.mark.parametrize("sizes,window", [([(1, 100), (6, 40)], 0), ([(150, 200), (40, 40)], 0), ([(150, 200)], 30)])
def test_what_a_row_does_not_see_does_not_reach_it(ctx, sizes, window):
    """Slots behind a sequence's end, positions behind a row's own and before its window, other rows of q: no numbers all of them."""
    case = Case(sizes, kv_heads=2, dim=128, page=32, seed=13)
    q = case.new(8, BF, size=2.0)
    want, tol = case.attention(q, window=window)
    nan = float("nan")
    dirty = torch.ones_like(case.k_scale, dtype=torch.bool)
    for b, (n, length) in enumerate(sizes):
        at, slot = case.places(b, 0, length)
        dirty[at, :, slot] = False
    case.k_scale[dirty] = nan
    case.v_scale[dirty] = nan
    got = ctx.kv_attend(case.cache, case.batch, q, window=window)
    assert ((got.double() - want).abs() <= tol).all()
    # the newest position of the first sequence is no number: of its rows the last alone sees it
    n, length = sizes[0]
    at, slot = case.places(0, length - 1, length)
    case.k_scale[at, :, slot] = nan
    got = ctx.kv_attend(case.cache, case.batch, q, window=window)
    assert torch.isnan(got[n - 1]).all()
    keep = [i for i in range(case.rows) if i != n - 1]
    assert ((got.double() - want).abs() <= tol)[keep].all()
    case.k_scale[at, :, slot] = 0.01
    # a row of q that is none
    q[-1, 3] = nan
    q[-1, 5] = float("inf")
    got = ctx.kv_attend(case.cache, case.batch, q, window=window)
    assert torch.isnan(got[-1, 3]).all() and torch.isnan(got[-1, 5]).all()
    want, tol = case.attention(q.nan_to_num(0.0, 0.0, 0.0), window=window)
    ok = (got.double() - want).abs() <= tol
    ok[-1, 3] = ok[-1, 5] = True
    assert ok.all()


@pytest.mark.parametrize("n", [7, 60])
def test_rows_of_padding_are_zeros_and_rows_behind_are_left(ctx, n):
    case = Case([(n, 3), (2, 40)], kv_heads=1, dim=64, page=16)
    q = case.new(4, BF, rows=n + 6)
    out = torch.full((n + 6, 4, 64), 9.0, dtype=BF, device=DEV)
    ctx.kv_attend(case.cache, case.batch, q, out=out)
    want, tol = case.attention(q[:n + 2])
    assert (out[:n - 3] == 0).all() and (out[n + 2:] == 9.0).all()
    assert ((out[:n + 2].double() - want).abs() <= tol).all()
    # a sequence without positions
    case.lengths.zero_()
    ctx.kv_attend(case.cache, case.batch, q, out=out)
    assert (out[:n + 2] == 0).all() and (out[n + 2:] == 9.0).all()


@pytest.mark.parametrize("sizes", [[(1, 70), (3, 20)], [(90, 100)]])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_rows_of_wider_arrays(ctx, sizes, shift):
    case = Case(sizes, kv_heads=2, dim=64, page=16, seed=4)
    fused = torch.randn(case.rows, 12 * 64 + 40, generator=case.gen, device=DEV).to(HF)
    q = fused[:, 16 + shift:16 + shift + 512].view(case.rows, 8, 64)
    wide = torch.full((case.rows, 8 * 64 + 40), 5.0, dtype=HF, device=DEV)
    out = wide[:, 24 + shift:24 + shift + 512].view(case.rows, 8, 64)
    check(ctx, case, q, out=out)
    wide[:, 24 + shift:24 + shift + 512] = 5.0
    assert (wide == 5.0).all()
    # one row of q for all heads
    same = q[:, :1].expand(-1, 8, -1)
    check(ctx, case, same)


@pytest.mark.parametrize("sizes", [[(1, 3000), (1, 100)], [(300, 5000)], [(1, 100), (40, 900)]])
def test_runs_give_the_same_bits(ctx, sizes):
    case = Case(sizes, kv_heads=2, dim=128, page=64, seed=6)
    q = case.new(8, BF, size=2.0)
    first = ctx.kv_attend(case.cache, case.batch, q)
    for _ in range(5):
        assert torch.equal(ctx.kv_attend(case.cache, case.batch, q), first)


def test_a_small_workspace_cuts_less():
    """A context of 64 x 64 holds two parts of few rows and none of a tile."""
    case = Case([(1, 2000), (1, 900), (70, 700)], kv_heads=2, dim=128, page=16, seed=8)
    q = case.new(8, BF, size=2.0)
    want, tol = case.attention(q)
    for d in (64, 128, 256, 512):
        c = Bd.ArmorContext(d, d, 32, device=DEV, h_mode=Bd.H_DIAG)
        got = c.kv_attend(case.cache, case.batch, q)
        assert ((got.double() - want).abs() <= tol).all() and c.device_status()[2] == 0
        c.close()


def test_pages_out_of_range_are_refused():
    c = Bd.ArmorContext(256, 256, 32, device=DEV)
    for sizes in ([(1, 200), (1, 50)], [(100, 200), (50, 50)]):
        case = Case(sizes, kv_heads=2, dim=64, page=16, seed=1)
        q = case.new(4, BF)
        want, tol = case.attention(q)
        before = c.device_status()[11]
        case.pages[0, 3] = 10 ** 7
        got = c.kv_attend(case.cache, case.batch, q)
        n = sizes[0][0]
        assert ((got.double() - want).abs() <= tol)[n:].all() and torch.isfinite(got).all()
        assert c.device_status()[11] > before and c.device_status()[3] == 1 and c.device_status()[2] == 0
        # offsets out of order and out of range, positions behind the table
        out = torch.full_like(q, 4.0)
        case.starts.copy_(torch.tensor([5, 2, 10 ** 6], dtype=torch.int32))
        case.lengths.fill_(10 ** 6)
        c.kv_attend(case.cache, case.batch, q, out=out)
        assert (out == 4.0).all()
        case.starts.copy_(torch.tensor([0, 1, 2], dtype=torch.int32))
        c.kv_attend(case.cache, case.batch, q, out=out)
        assert torch.isfinite(out).all()
    c.close()


def test_cache_of_more_than_2_31_bytes(ctx):
    page, heads, dim = 256, 8, 128
    n = (2 ** 31) // (page * heads * dim) + 3
    cache = ctx.new_kv_cache(n, page, heads, dim)
    small = Case([(1, 400), (90, 400)], kv_heads=heads, dim=dim, page=page, seed=5, spare=0)
    far = torch.arange(n - 4, n, device=DEV).int().view(2, 2)
    for t in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, t)[far.flatten().long()] = getattr(small, t)[small.pages.flatten().long()]
    q = small.new(16, BF, size=2.0)
    got = ctx.kv_attend(cache, Bd.KvBatch(far, small.lengths, small.starts), q)
    want, tol = small.attention(q)
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("sizes", [[(1, 60), (1, 1000)], [(1, 60), (33, 1000)]])
def test_a_captured_step_follows_the_batch(ctx, sizes):
    """A decoding step in a graph, the new keys written and looked at in it; lengths grow between replays."""
    case = Case([(n, length + 8) for n, length in sizes], kv_heads=2, dim=128, page=16, seed=17)
    case.lengths -= 8
    case.sizes = list(sizes)
    q, k, v = case.new(8, BF), case.new(2, BF), case.new(2, BF)
    out = torch.empty_like(q)
    ctx.kv_attend(case.cache, case.batch, q, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.kv_write(case.cache, case.batch, k, v)
        ctx.kv_attend(case.cache, case.batch, q, out=out)
    for step in range(4):
        case.lengths += 2
        case.sizes = [(n, length + 2) for n, length in case.sizes]
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=case.gen, device=DEV))
        g.replay()
        want, tol = case.attention(q)
        assert ((out.double() - want).abs() <= tol).all()


def test_two_contexts_side_by_side():
    """Contexts of their own on two streams, many calls under way at once; one context's calls follow each other on a stream that is not the default."""
    cases = [Case([(1, 5000), (1, 300)], kv_heads=2, dim=128, page=16, seed=1), Case([(200, 900)], kv_heads=2, dim=128, page=16, seed=2)]
    contexts = [Bd.ArmorContext(512, 512, 32, device=DEV, h_mode=Bd.H_DIAG) for _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    qs = [c.new(8, BF, size=2.0) for c in cases]
    alone = [ctx.kv_attend(c.cache, c.batch, q) for ctx, c, q in zip(contexts, cases, qs)]
    outs = [[torch.empty_like(q) for _ in range(20)] for q in qs]
    torch.cuda.synchronize()
    for i in range(20):
        for ctx, c, q, s, o in zip(contexts, cases, qs, streams, outs):
            with torch.cuda.stream(s):
                ctx.kv_attend(c.cache, c.batch, q, out=o[i])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, x) for x in o)
    for ctx in contexts:
        assert ctx.device_status()[2] == 0
        ctx.close()


def test_two_captured_calls_of_one_context(ctx):
    """Graphs that share the workspace, replayed one after the other."""
    cases = [Case([(1, 9000)], kv_heads=2, dim=128, page=16, seed=1), Case([(60, 9000)], kv_heads=2, dim=128, page=16, seed=2)]
    qs = [c.new(8, HF, size=2.0) for c in cases]
    outs, graphs = [torch.empty_like(q) for q in qs], []
    want = [ctx.kv_attend(c.cache, c.batch, q) for c, q in zip(cases, qs)]
    torch.cuda.synchronize()
    for c, q, o in zip(cases, qs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.kv_attend(c.cache, c.batch, q, out=o)
        graphs.append(g)
    for _ in range(3):
        for g, o, w in zip(graphs, outs, want):
            o.zero_()
            g.replay()
            assert torch.equal(o, w)


def test_a_block_of_a_served_model(ctx):
    """Norm, 8-bit products for q, k and v, the cache, the attention, the output's product and the next norm: a prompt, then three decoding steps, against the
    whole prompt at once in the same calls, and against 64 bits from what each call was given."""
    d, kv_heads, dim, group, page = 1024, 2, 128, 4, 16
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    w_qkv, w_o = (torch.randn(n, m, generator=gen, device=DEV) * 0.03 for n, m in (((group + 2) * kv_heads * dim, d), (d, group * kv_heads * dim)))
    (qkv_q, qkv_s), (o_q, o_s) = ctx.quantize_rows(w_qkv), ctx.quantize_rows(w_o)
    w_pre = 1.0 + 0.1 * torch.randn(d, generator=gen, device=DEV)
    x = torch.randn(13, d, generator=gen, device=DEV).bfloat16()
    heads = group * kv_heads

    def run(cache, batch, rows):
        _, nq, ns = ctx.block_norm_i8(rows, w_pre=w_pre)
        fused = ctx.linear_i8(nq, qkv_q, qkv_s, x_scale=ns).view(rows.shape[0], heads + 2 * kv_heads, dim)
        ctx.kv_write(cache, batch, fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:])
        o = ctx.kv_attend(cache, batch, fused[:, :heads])
        y = ctx.linear_i8(o.view(rows.shape[0], -1), o_q, o_s)
        return fused, o, ctx.block_norm(rows, y, w_pre=w_pre)

    case = Case([(13, 13)], kv_heads=kv_heads, dim=dim, page=page)
    fused, o, (h, n) = run(case.cache, case.batch, x)
    want, tol = case.attention(fused[:, :heads])
    assert ((o.double() - want).abs() <= tol).all()
    # the same tokens a prompt of ten and three single ones: the same cache, exactly, and the same attention within its rounding
    steps = Case([(10, 10)], kv_heads=kv_heads, dim=dim, page=page, seed=1)
    got = [run(steps.cache, steps.batch, x[:10])]
    for i in (10, 11, 12):
        steps.lengths.fill_(i + 1)
        steps.starts.copy_(torch.tensor([0, 1], dtype=torch.int32))
        got.append(run(steps.cache, steps.batch, x[i:i + 1]))
    assert torch.equal(torch.cat([g[0] for g in got]), fused)
    at, slot = case.places(0, 0, 13)
    at2, slot2 = steps.pages[0].long()[torch.arange(13, device=DEV) // page], torch.arange(13, device=DEV) % page
    for t in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(case, t)[at, :, slot], getattr(steps, t)[at2, :, slot2])
    assert ((torch.cat([g[1] for g in got]).double() - want).abs() <= tol).all()
    assert torch.isfinite(torch.cat([g[2][0] for g in got])).all() and torch.isfinite(h).all() and torch.isfinite(n).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [1, 16, 17, 48, 64])
@pytest.mark.parametrize("sizes", [[(1, 300), (1, 50)], [(100, 300), (20, 50)]])
def test_only_the_positions_of_a_page_that_is_not_there_are_missed(sizes, page, dim):
    with_status = Bd.ArmorContext(256, 256, 32, device=DEV)
    case = Case(sizes, kv_heads=2, dim=dim, page=page, seed=2)
    q = case.new(6, BF, size=2.0)
    at = 70 // page
    want, tol = case.attention(q, gone=slice(at * page, (at + 1) * page))
    case.pages[0, at] = -1
    got = with_status.kv_attend(case.cache, case.batch, q)
    assert ((got.double() - want).abs() <= tol).all()
    assert with_status.device_status()[11] > 0
    with_status.close()


@pytest.mark.parametrize("page", [1, 16, 17, 48, 64])
@pytest.mark.parametrize("sizes", [[(1, 700), (1, 500)], [(100, 700), (20, 500)]])
def test_pages_before_a_window_may_be_gone(ctx, sizes, page):
    """(and count as none that is refused: the fixture looks)"""
    case = Case(sizes, kv_heads=2, dim=64, page=page, seed=3)
    q = case.new(6, BF, size=2.0)
    window = 150
    want = check(ctx, case, q, window=window)
    for b, (n, length) in enumerate(sizes):
        case.pages[b, :(length - n + 1 - window) // page] = -1
    assert torch.equal(ctx.kv_attend(case.cache, case.batch, q, window=window), want)


@pytest.mark.parametrize("chunk", [1, 40])
def test_a_sequence_too_long_for_any_call_is_refused(chunk):
    c = Bd.ArmorContext(256, 256, 32, device=DEV)
    cache = c.new_kv_cache(1, 4096, 1, 64)
    batch = Bd.KvBatch(torch.zeros(1, 2 ** 19, dtype=torch.int32, device=DEV), torch.tensor([2 ** 31 - 4095], dtype=torch.int32, device=DEV),
                       torch.tensor([0, chunk], dtype=torch.int32, device=DEV))
    k = torch.ones(chunk, 1, 64, dtype=BF, device=DEV)
    c.kv_write(cache, batch, k, k)
    assert (cache.k == 0).all() and (c.kv_read(cache, batch, chunk)[0] == 0).all()
    out = torch.full_like(k, 4.0)
    before = c.device_status()[11]
    c.kv_attend(cache, batch, k, out=out)
    assert (out == 4.0).all() and c.device_status()[11] > before
    c.close()


def test_a_hint_of_any_size(ctx):
    case = Case([(5, 300), (1, 50)], kv_heads=2, dim=64, page=16, seed=4)
    check(ctx, case, case.new(8, BF), max_chunk=2 ** 62)


def test_binding_refuses(ctx):
    case = Case([(2, 20)], kv_heads=2, dim=64, page=16)
    cache, batch, q = case.cache, case.batch, case.new(4, BF)

    def refused(match, f, *args, **kw):
        with pytest.raises(ValueError, match=match):
            f(*args, **kw)

    k, s = torch.zeros(3, 2, 16, 64, dtype=torch.int8, device=DEV), torch.zeros(3, 2, 16, device=DEV)
    for args, match in [((k.float(), k, s, s), "int8"), ((k, k, s, s.half()), "float32"), ((k[:2], k, s, s), r"\[2, 2, 16, 64\]"),
                        ((k, k, s[:, :1], s), r"\[3, 2, 16\]"), ((k, k.transpose(1, 2).contiguous().transpose(1, 2), s, s), "alike"),
                        ((k, k, s, s.transpose(1, 2).contiguous().transpose(1, 2)), "alike"), ((k[:0], k[:0], s[:0], s[:0]), "hold a page"),
                        ((k, k.expand(3, 2, 16, 64)[..., ::1].cpu(), s, s), "CUDA"), ((k[:, :1].expand(3, 2, 16, 64),) * 2 + (s, s), "overlap")]:
        refused(match, Bd.KvCache, *args)
    wide = torch.zeros(3, 2, 16, 80 + 8, dtype=torch.int8, device=DEV)
    refused("16-byte", Bd.KvCache, wide[..., :64], wide[..., :64], s, s)
    refused("16-byte", Bd.KvCache, wide[..., 8:72], wide[..., 8:72], s, s)
    refused("contiguous", Bd.KvCache, k.transpose(2, 3), k.transpose(2, 3), torch.zeros(3, 2, 64, device=DEV), torch.zeros(3, 2, 64, device=DEV))

    pages, lengths, starts = case.pages, case.lengths, case.starts
    for args, match in [((pages.long(), lengths, starts), "int32"), ((pages, lengths, starts[:1]), "2 starts"), ((pages, starts, starts), "1 lengths"),
                        ((pages[0], lengths, starts), "2 dimensions"), ((pages, lengths, starts.cpu()), "CUDA"),
                        ((pages.repeat(2, 1).T.contiguous().T, starts, torch.zeros(3, dtype=torch.int32, device=DEV)), "contiguous")]:
        refused(match, Bd.KvBatch, *args)

    refused("dtype", ctx.kv_attend, cache, batch, q.float(), out=q)
    with pytest.raises(Bd.ArmorError):
        ctx.kv_attend(cache, batch, q.float())
    with pytest.raises(Bd.ArmorError):                      # heads that share no whole groups
        ctx.kv_attend(cache, batch, case.new(3, BF))
    for kw in ({"window": -1}, {"max_chunk": -1}, {"scale": -1.0}, {"scale": float("nan")}):
        with pytest.raises(Bd.ArmorError):
            ctx.kv_attend(cache, batch, q, **kw)
    refused("rows, heads, 64", ctx.kv_attend, cache, batch, q[..., :32])
    refused(r"\[2, 4, 64\]", ctx.kv_attend, cache, batch, q, out=q[:1])
    refused("dtype", ctx.kv_attend, cache, batch, q, out=q.half())
    refused("CUDA", ctx.kv_attend, cache, batch, q, out=q.cpu())
    refused("CUDA", ctx.kv_attend, cache, batch, q.cpu())
    new = case.new(2, BF)
    refused("2, 64", ctx.kv_write, cache, batch, q, q)
    refused("dtype", ctx.kv_write, cache, batch, new, new.half())
    refused(r"\[2, 2, 64\]", ctx.kv_write, cache, batch, new, new[:1])
    refused("2 rows", ctx.kv_read, cache, batch, 2, BF, out=(new[:1], new[:1]))
    refused("float16", ctx.kv_read, cache, batch, 2, torch.float16, out=(new, new))
    with pytest.raises((ValueError, Bd.ArmorError)):
        ctx.kv_read(cache, batch, 2, torch.float64)
    with pytest.raises((ValueError, Bd.ArmorError)):        # rows that overlap are not written
        ctx.kv_read(cache, batch, 2, BF, out=(new[:1].expand(2, 2, 64), new))


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 17), (128, 64)])
@pytest.mark.parametrize("group,max_chunk", [(1, 0), (1, 33), (4, 0), (8, 0), (17, 0), (32, 1), (33, 0)])
def test_rows_on_either_side_of_a_choice_of_kernels(ctx, group, max_chunk, dim, page):
    case = Case([(n, 37 + 61 * n) for n in (1, 2, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33)], kv_heads=2, dim=dim, page=page, seed=6)
    check(ctx, case, case.new(2 * group, BF), max_chunk=max_chunk)
    one = Case([(4, 300)], kv_heads=2, dim=dim, page=page, seed=7)
    check(ctx, one, one.new(2 * group, BF), max_chunk=max_chunk)
