"""The paged cache's calls where no GPU is needed: what is refused by sizes and types, which are looked at before the context; the C layout; the rules
of kernels that start while the one before them runs."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from paper_2510_05528_b200 import build as armor_build
from tests.test_dependent_launches import LAUNCHED, TEXT

INVALID, SHAPE, UNSUPPORTED, TOO_LARGE = 1, 2, 7, 8
P = 0x10000
CACHE = {"k": P, "v": P, "k_scale": P, "v_scale": P, "n_pages": 4, "page_size": 16, "kv_heads": 2, "head_dim": 64, "page_stride": 2048,
         "head_stride": 1024, "slot_stride": 64, "scale_page_stride": 32, "scale_head_stride": 16, "scale_slot_stride": 1}
BATCH = {"n_seqs": 2, "max_pages": 3, "ld_pages": 3, "pages": P, "lengths": P, "starts": P}
ROWS = {"k": P, "v": P, "n_rows": 5, "k_row_stride": 128, "k_head_stride": 64, "v_row_stride": 128, "v_head_stride": 64, "dtype": Bd.DTYPE_BF16}
ATTEND = {"q": P, "o": P, "n_rows": 5, "heads": 8, "q_row_stride": 512, "q_head_stride": 64, "o_row_stride": 512, "o_head_stride": 64, "scale": 0.125,
          "dtype": Bd.DTYPE_BF16}
ANY = [
    (INVALID, {}, {}),                                        # no context
    (SHAPE, {"n_pages": 0}, {}), (SHAPE, {"page_size": 0}, {}), (SHAPE, {"kv_heads": 0}, {}), (UNSUPPORTED, {"head_dim": 96}, {}),
    (TOO_LARGE, {"n_pages": 2 ** 31}, {}), (TOO_LARGE, {"page_size": 2 ** 31}, {}), (SHAPE, {"slot_stride": 32}, {}), (SHAPE, {"slot_stride": 72}, {}),
    (SHAPE, {"page_stride": 2056}, {}), (SHAPE, {"head_stride": 0}, {}), (SHAPE, {"scale_slot_stride": 0}, {}), (SHAPE, {"k": P + 8}, {}),
    (SHAPE, {"v": P + 8}, {}), (INVALID, {"k_scale": None}, {}), (INVALID, {"v": None}, {}),
    (INVALID, {}, {"n_seqs": -1}), (SHAPE, {}, {"max_pages": -1}), (SHAPE, {}, {"ld_pages": 2}), (INVALID, {}, {"starts": None}),
    (INVALID, {}, {"pages": None}), (TOO_LARGE, {}, {"n_seqs": 2 ** 31}),
]


@pytest.fixture(scope="module")
def lib():
    armor_build.build()
    return Bd.lib()


@pytest.mark.parametrize("want,cache,batch", ANY)
@pytest.mark.parametrize("call,args", [("write", ROWS), ("read", ROWS), ("attend", ATTEND)])
def test_any_call_refuses(lib, call, args, want, cache, batch):
    g = (Bd.armor_kv_attend_args if call == "attend" else Bd.armor_kv_rows)(**args)
    f = getattr(lib, "armor_kv_" + call)
    assert f(None, Bd.armor_kv_cache(**{**CACHE, **cache}), Bd.armor_kv_batch(**{**BATCH, **batch}), g, None) == want
    c, b = Bd.armor_kv_cache(**CACHE), Bd.armor_kv_batch(**BATCH)
    assert f(None, None, b, g, None) == f(None, c, None, g, None) == f(None, c, b, None, None) == INVALID


@pytest.mark.parametrize("want,change", [
    (INVALID, {"n_rows": -1}), (UNSUPPORTED, {"dtype": Bd.DTYPE_I8}), (UNSUPPORTED, {"dtype": Bd.DTYPE_BF16_SPARSE}), (SHAPE, {"k_row_stride": -1}),
    (SHAPE, {"v_head_stride": -64}), (TOO_LARGE, {"n_rows": 2 ** 31}),
])
def test_rows_refused(lib, want, change):
    for call in ("write", "read"):
        assert getattr(lib, "armor_kv_" + call)(None, Bd.armor_kv_cache(**CACHE), Bd.armor_kv_batch(**BATCH), Bd.armor_kv_rows(**{**ROWS, **change}), None) == want


@pytest.mark.parametrize("change", [{"k_row_stride": 63}, {"k_head_stride": 0}, {"v_row_stride": 0}, {"v_head_stride": 32}])
def test_outputs_must_not_overlap(lib, change):
    args = Bd.armor_kv_rows(**{**ROWS, **change})
    assert lib.armor_kv_read(None, Bd.armor_kv_cache(**CACHE), Bd.armor_kv_batch(**BATCH), args, None) == SHAPE


@pytest.mark.parametrize("want,change", [
    (INVALID, {"n_rows": -1}), (UNSUPPORTED, {"dtype": Bd.DTYPE_F32}), (SHAPE, {"heads": 0}), (SHAPE, {"heads": 7}), (SHAPE, {"q_row_stride": -1}),
    (SHAPE, {"o_row_stride": 63}), (SHAPE, {"o_head_stride": 0}), (INVALID, {"window": -1}), (INVALID, {"max_chunk": -1}), (INVALID, {"scale": -1.0}),
    (INVALID, {"scale": float("nan")}), (INVALID, {"scale": float("inf")}), (TOO_LARGE, {"n_rows": 2 ** 29, "heads": 16}),
])
def test_attend_refuses(lib, want, change):
    args = Bd.armor_kv_attend_args(**{**ATTEND, **change})
    assert lib.armor_kv_attend(None, Bd.armor_kv_cache(**CACHE), Bd.armor_kv_batch(**BATCH), args, None) == want


def test_structs_are_laid_out_as_in_the_header(lib, tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = (Bd.armor_kv_cache, Bd.armor_kv_batch, Bd.armor_kv_rows, Bd.armor_kv_attend_args)
    lines = []
    for s in structs:
        lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for f, _ in s._fields_] + [f'printf("%zu\\n", sizeof({s.__name__}));']
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "armor.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "layout")]).split()]
    want = []
    for s in structs:
        want += [getattr(s, f).offset for f, _ in s._fields_] + [C.sizeof(s)]
    assert got == want


def test_binding_refuses():
    k, s = torch.zeros(2, 1, 16, 64, dtype=torch.int8), torch.zeros(2, 1, 16)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.KvCache(k, k, s, s)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.KvBatch(torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_division_by_the_page_size():
    """quotient(p) = p mul >> shift with the reciprocal that divisor() forms, at the borders where it could be off."""
    for d in [*range(1, 600), 1000, 4096, 65535, 65537, 2 ** 20 + 1, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 1]:
        s = 0
        while (1 << s) < d:
            s += 1
        mul, shift = ((1 << (31 + s)) + d - 1) // d, 31 + s
        assert mul < 2 ** 32
        top = (2 ** 31 - 1) // d * d
        for p in {0, 1, d - 1, d, d + 1, top - 1, top, min(top + d - 1, 2 ** 31 - 1), 2 ** 31 - 1, 2 ** 30, 123456789}:
            if 0 <= p < 2 ** 31:
                assert (p * mul) >> shift == p // d
                assert p * mul < 2 ** 64


def test_every_launch_of_these_files_is_a_dependent_one():
    """So that the rules of tests/test_dependent_launches.py are looked at for all of their kernels."""
    for f in [n for n in TEXT if n.startswith("kv_") and n.endswith(".cu")]:
        kernels = {re.search(r"(\w+_kernel)\s*\(", TEXT[f][m.end():]).group(1) for m in re.finditer("__global__", TEXT[f])}
        assert kernels and kernels == {k for g, k in LAUNCHED if g == f}
        assert "<<<" not in TEXT[f]
