"""The packed layer with an int8 core rounds z1 to int8 and y to bf16, and nothing between to fewer than 15 bits: z2 goes to the product with A as
two bf16 numbers.

Bound: with B the identity and tokens of whole numbers whose largest is 127, z1 and its integers are exact, and z2 = ws[m] times an integer, two
roundings to fp32.  Its bf16 number is off by at most 2^-8 of it, the rest's bf16 number, rounded towards zero, by less than 2^-7 of the rest:
2^-15.  A's blocks are bf16 already.  A sum of 2 d_block <= 512 products in fp32, each addition off by 2^-23 at most if it truncates:
2^-14.  Together less than 2^-13 of sum |A| |z2|; then the half step of y."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.test_gpu_int8 import BF16, DEV, HALF_STEP, gen, layer, quantized

pytestmark = pytest.mark.gpu


def near_exact(d_out, d_in, db, n, seed):
    c = Bd.ArmorContext(d_out, d_in, db, device=DEV)
    st = layer(c, d_out, d_in, db, seed)
    st.B = torch.eye(db, device=DEV).repeat(d_in // db, 1, 1)
    x = torch.randint(-126, 127, (n, d_in), generator=gen(n + seed), device=DEV).float()
    x[torch.arange(n, device=DEV), torch.arange(n, device=DEV) % d_in] = 127.0
    Sq, Ss = quantized(st.S)
    z2 = (x.double() @ Sq.double().t()) * Ss.double()
    want = torch.einsum("tjk,jmk->tjm", z2.view(n, -1, db), st.A.double()).reshape(n, d_out)
    size = torch.einsum("tjk,jmk->tjm", z2.abs().view(n, -1, db), st.A.double().abs()).reshape(n, d_out)
    return c, st, x, want, size


def check(y, want, size):
    err = 2.0 ** -13 * size
    assert ((y.double() - want).abs() <= err + HALF_STEP[BF16] * (want.abs() + err)).all()


@pytest.mark.parametrize("d_out,d_in,db", [(256, 256, 128), (384, 640, 128), (512, 768, 256), (2048, 1024, 128), (1024, 2048, 256)])
@pytest.mark.parametrize("n", [1, 2, 3, 17, 128, 200, 600, 1500, 9000])
def test_y_is_rounded_once(d_out, d_in, db, n):
    c, st, x, want, size = near_exact(d_out, d_in, db, n, 11)
    y = c.apply_layer_i8(c.pack_layer_i8(st), x.to(BF16))
    check(y, want, size)
    assert c.device_status()[:4] == [0, 0, 0, 0]


def test_in_chunks_and_in_a_graph():
    """More tokens than the workspace takes at once, with nothing written behind the last; and replayed on other tokens."""
    c, st, x, want, size = near_exact(256, 512, 128, 5000, 12)
    packed = c.pack_layer_i8(st)
    buf = torch.full((5004, 256), 3.0, dtype=BF16, device=DEV)
    Bd.armor_apply_layer_i8(c.ctx, packed, x.to(BF16), buf[:5000])
    check(buf[:5000], want, size)
    assert (buf[5000:] == 3.0).all()
    held = x.to(BF16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = c.apply_layer_i8(packed, held)
    held.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, buf[:5000].flip(0))


@pytest.mark.parametrize("n", [5, 300])
def test_values_at_the_ends_of_the_range(n):
    """z2 that only bf16 cannot hold is an infinity of its sign, as one rounding to bf16 makes it, and no NaN."""
    d = 256
    c = Bd.ArmorContext(d, d, 128, device=DEV)
    eye = torch.eye(128, device=DEV).repeat(2, 1, 1)
    # a row of the core keeps its first entry alone: z2 = +- that entry
    value = torch.exp2(torch.linspace(-100, 126, d, device=DEV).round())
    value[-1] = (2 - 2.0 ** -9) * 2.0 ** 127
    S = torch.zeros(d, d, device=DEV)
    S[:, 0] = value
    M = torch.full((d, d // 4), 3, dtype=torch.uint8, device=DEV)
    packed = c.pack_layer_i8(Bd.LayerState(Wbar=S, A=eye, B=eye, S=S, M=M))
    x = torch.zeros(n, d, device=DEV)
    x[:, 0] = 1.0
    x[::2, 0] = -1.0
    y = c.apply_layer_i8(packed, x.to(BF16))
    z2 = x[:, :1].double() * value.double()
    assert ((y[:, :128].double() - z2[:, :128]).abs() <= (HALF_STEP[BF16] + 2.0 ** -20) * z2[:, :128].abs()).all()
    assert torch.equal(y[:, -1], z2[:, -1].to(BF16)) and y[:, -1].isinf().all()
