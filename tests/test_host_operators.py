"""The 8-bit products and the norms where no GPU is needed: their sizes, and calls that are refused by what they ask for.  The sizes and
types of a call are looked at before its context."""
import ctypes as C

import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from paper_2510_05528_b200 import build as armor_build

INVALID, SHAPE, UNSUPPORTED, TOO_LARGE = 1, 2, 7, 8
F32, BF16, SPARSE, F16, I8 = Bd.DTYPE_F32, Bd.DTYPE_BF16, Bd.DTYPE_BF16_SPARSE, Bd.DTYPE_F16, Bd.DTYPE_I8


@pytest.fixture(scope="module")
def lib():
    armor_build.build()
    return Bd.lib()


def at(n=0x10000):
    return C.c_void_p(n)


@pytest.mark.parametrize("want,change", [
    (INVALID, {}),                                         # no context
    (INVALID, {"n_rows": -1}), (UNSUPPORTED, {"x_dtype": SPARSE}), (UNSUPPORTED, {"x_dtype": I8}), (UNSUPPORTED, {"x_dtype": 9}),
    (SHAPE, {"n_cols": 0}), (SHAPE, {"ldx": 99}), (SHAPE, {"ldq": 100}), (SHAPE, {"ldq": 96}), (SHAPE, {"q": at(0x10008)}),
])
def test_quantize_rows_refuses(lib, want, change):
    a = {"x": at(), "x_dtype": F32, "ldx": 100, "n_rows": 4, "n_cols": 100, "q": at(), "ldq": 112, "scale": at(), **change}
    assert lib.armor_quantize_rows(None, a["x"], a["x_dtype"], a["ldx"], a["n_rows"], a["n_cols"], a["q"], a["ldq"], a["scale"], None) == want


@pytest.mark.parametrize("want,change", [
    (INVALID, {}), (INVALID, {"n_tokens": -1}),
    (UNSUPPORTED, {"x_dtype": SPARSE}), (UNSUPPORTED, {"x_dtype": -1}), (UNSUPPORTED, {"y_dtype": I8}), (UNSUPPORTED, {"y_dtype": SPARSE}),
    (SHAPE, {"n_out": 0}), (SHAPE, {"n_in": 0}), (SHAPE, {"ldx": 99}), (SHAPE, {"ldw": 96}), (SHAPE, {"ldw": 104}), (SHAPE, {"ldy": 49}),
    (SHAPE, {"x_dtype": I8, "ldx": 100}), (SHAPE, {"w": at(0x10004)}), (SHAPE, {"x_dtype": I8, "ldx": 112, "x": at(0x10008)}),
    (TOO_LARGE, {"n_in": 131072, "ldx": 131072, "ldw": 131072}), (TOO_LARGE, {"n_tokens": 2 ** 30 + 1}),
    (TOO_LARGE, {"n_out": 2 ** 30 + 1, "ldy": 2 ** 30 + 1}),
])
def test_linear_i8_refuses(lib, want, change):
    a = {"x": at(), "x_dtype": BF16, "ldx": 100, "xs": None, "w": at(), "ldw": 112, "ws": at(), "y": at(), "y_dtype": BF16, "ldy": 50, "n_tokens": 3,
         "n_out": 50, "n_in": 100, **change}
    assert lib.armor_linear_i8(None, a["x"], a["x_dtype"], a["ldx"], a["xs"], a["w"], a["ldw"], a["ws"], None, a["y"], a["y_dtype"], a["ldy"],
                               a["n_tokens"], a["n_out"], a["n_in"], None) == want


def test_packed_layer_i8_sizes(lib):
    """Kept values (half the entries), positions (4 bits a group, in stages of 256 k and tiles of 256 rows), bf16 wrappers, scales."""
    for d_out, d_in, db in ((512, 768, 128), (512, 768, 256), (384, 640, 128)):
        rows, k = -(-d_out // 256) * 256, -(-d_in // 256) * 256
        want = d_out * d_in // 2 + rows * k // 8 + (d_out + d_in) * db * 2 + d_out * 4
        assert Bd.armor_packed_layer_i8_bytes(Bd.make_config(d_out, d_in, db)) == want
    n = C.c_size_t(0)
    for bad in (Bd.make_config(512, 768, 128, n_keep=4, m_group=8), Bd.make_config(512, 704, 64), Bd.make_config(512, 768, 64)):
        assert lib.armor_packed_layer_i8_bytes(C.byref(bad), C.byref(n)) == UNSUPPORTED
    assert lib.armor_packed_layer_i8_bytes(None, C.byref(n)) == INVALID
    assert lib.armor_packed_layer_i8_bytes(C.byref(Bd.make_config(512, 768, 128)), None) == INVALID
    assert lib.armor_pack_layer_i8(None, *[None] * 8) == INVALID
    assert lib.armor_apply_layer_i8(None, None, None, None, 4, None) == INVALID


P = 0x10000
NORM = {"n_rows": 6, "d": 64, "x": P, "ldx": 64, "y": P, "ldy": 64, "h": P, "ldh": 64, "n": P, "ldn": 64, "stream_dtype": BF16,
        "branch_dtype": BF16, "pre": 1, "post": 1, "residual_scale": 1.0, "eps": 1e-6}
GRAD = {"n_rows": 6, "d": 64, "h": P, "ldh": 64, "y": P, "ldy": 64, "dh": P, "lddh": 64, "dn": P, "lddn": 64, "dx": P, "lddx": 64, "dy": P,
        "lddy": 64, "stream_dtype": BF16, "branch_dtype": BF16, "pre": 1, "post": 1, "residual_scale": 1.0, "eps": 1e-6}
GATE = {"gate": P, "ld_gate": 64, "rows_per_gate": 3, "n_gates": 2}
BOTH = [
    (INVALID, {}), (INVALID, {"n_rows": -1}), (INVALID, {"eps": -1.0}), (INVALID, {"eps": float("nan")}), (SHAPE, {"d": 0}),
    (TOO_LARGE, {"d": 16385}), (TOO_LARGE, {"n_rows": 2 ** 31}),
    (UNSUPPORTED, {"stream_dtype": SPARSE}), (UNSUPPORTED, {"branch_dtype": I8}), (UNSUPPORTED, {"branch_dtype": F32}),
    (UNSUPPORTED, {"stream_dtype": F16}), (SHAPE, {"ldy": 63}), (SHAPE, {"ldh": 63}),
    (SHAPE, {**GATE, "n_gates": 1}), (SHAPE, {**GATE, "rows_per_gate": 0}), (SHAPE, {**GATE, "ld_gate": 63}), (SHAPE, {**GATE, "n_gates": 0}),
    (INVALID, {"w_pre": P, "pre": 0}), (INVALID, {"w_post": P, "post": 0}), (INVALID, GATE),
]


@pytest.mark.parametrize("want,change", BOTH + [
    (INVALID, {"y": None}), (INVALID, {"y": None, "post": 0, **GATE}), (SHAPE, {"ldx": 63}), (SHAPE, {"ldn": 63}),
    (SHAPE, {"q": P, "q_scale": P, "ldq": 72}), (SHAPE, {"q": P + 8, "q_scale": P, "ldq": 64}), (SHAPE, {"q": P, "q_scale": P, "ldq": 48}),
    (INVALID, {"q": P, "ldq": 64}),
])
def test_block_norm_refuses(lib, want, change):
    assert lib.armor_block_norm(None, Bd.armor_block_norm_args(**{**NORM, **change}), None) == want
    assert lib.armor_block_norm(None, None, None) == INVALID


@pytest.mark.parametrize("want,change", BOTH + [
    (SHAPE, {"lddh": 63}), (SHAPE, {"lddn": 63}), (SHAPE, {"lddx": 63}), (SHAPE, {"lddy": 63}),
    (INVALID, {"dw_pre": P, "pre": 0}), (INVALID, {"dw_post": P, "post": 0}), (INVALID, {"dgate": P}),
])
def test_block_norm_backward_refuses(lib, want, change):
    assert lib.armor_block_norm_backward(None, Bd.armor_block_norm_grad_args(**{**GRAD, **change}), None) == want
    assert lib.armor_block_norm_backward(None, None, None) == INVALID


def test_structs_are_laid_out_as_in_the_header(lib, tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for s in (Bd.armor_block_norm_args, Bd.armor_block_norm_grad_args):
        lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for f, _ in s._fields_] + [f'printf("%zu\\n", sizeof({s.__name__}));']
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "armor.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "layout")]).split()]
    want = []
    for s in (Bd.armor_block_norm_args, Bd.armor_block_norm_grad_args):
        want += [getattr(s, f).offset for f, _ in s._fields_] + [C.sizeof(s)]
    assert got == want


def test_binding_refuses(lib):
    x = torch.zeros(4, 32)
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_quantize_rows(None, x, q, s)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        Bd.armor_quantize_rows(None, x.double(), q, s)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_linear_i8(None, x, None, q, s, None, x)
    with pytest.raises(ValueError, match="bf16"):
        Bd.armor_apply_layer_i8(None, q, x, x)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm(None, x, x, x, x, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.armor_block_norm_backward(None, x, x, x, x, x, x, None, None, None)
    with pytest.raises(ValueError, match="missing"):
        Bd.armor_block_norm_backward(None, None, None, None, None, None, None, None, None, None)
