"""Arrays of the paged cache's calls that do not lie on their elements' boundaries are refused (by their addresses, which are looked at before the context)."""
import pytest

from paper_2510_05528_b200 import binding as Bd
from tests.test_host_kv_cache import ATTEND, BATCH, CACHE, P, ROWS, SHAPE, INVALID, lib  # noqa: F401  (lib: a fixture)

CALLS = [("write", ROWS), ("read", ROWS), ("attend", ATTEND)]


def call(lib, name, args, cache=(), batch=(), change=()):
    g = (Bd.armor_kv_attend_args if name == "attend" else Bd.armor_kv_rows)(**{**args, **dict(change)})
    return getattr(lib, "armor_kv_" + name)(None, Bd.armor_kv_cache(**{**CACHE, **dict(cache)}), Bd.armor_kv_batch(**{**BATCH, **dict(batch)}), g, None)


@pytest.mark.parametrize("name,args", CALLS)
@pytest.mark.parametrize("off", [1, 2, 3])
def test_scales_and_the_arrays_of_a_batch(lib, name, args, off):
    for array in ("k_scale", "v_scale"):
        assert call(lib, name, args, cache={array: P + off}) == SHAPE
    for array in ("pages", "lengths", "starts"):
        assert call(lib, name, args, batch={array: P + off}) == SHAPE
    # on their boundary they are taken: what is missing is the context
    for array in ("k_scale", "v_scale"):
        assert call(lib, name, args, cache={array: P + 4}) == INVALID
    for array in ("pages", "lengths", "starts"):
        assert call(lib, name, args, batch={array: P + 4}) == INVALID


@pytest.mark.parametrize("dtype,size", [(Bd.DTYPE_BF16, 2), (Bd.DTYPE_F16, 2), (Bd.DTYPE_F32, 4)])
@pytest.mark.parametrize("name", ["write", "read"])
def test_rows(lib, name, dtype, size):
    for array in "kv":
        for off in (1, 2, 3, 4):
            assert call(lib, name, ROWS, change={array: P + off, "dtype": dtype}) == (SHAPE if off % size else INVALID)


@pytest.mark.parametrize("dtype", [Bd.DTYPE_BF16, Bd.DTYPE_F16])
def test_attend(lib, dtype):
    for array in "qo":
        for off in (1, 2, 3, 4):
            assert call(lib, "attend", ATTEND, change={array: P + off, "dtype": dtype}) == (SHAPE if off % 2 else INVALID)


def test_what_a_call_without_rows_does_not_read_is_not_looked_at(lib):
    for name, args in CALLS:
        none = {"lengths": None, "starts": None, "pages": None}
        assert call(lib, name, args, batch=none, change={"n_rows": 0}) == INVALID        # (no context)
        assert call(lib, name, args, batch={**none, "n_seqs": 0}) == INVALID
