"""The kernels of the 8-bit products and of the norms that are launched while the kernel before them may still run, where their launch
does not name them: the rules of tests/test_dependent_launches.py, read off the sources."""
import re

import pytest

from tests.test_dependent_launches import LAUNCHED, TEXT, _kernel, _only_written

WAITING = [("block_norm.cu", "block_norm_kernel"), ("block_norm.cu", "block_norm_ring_kernel"), ("block_norm.cu", "block_norm_grad_kernel"),
           ("block_norm.cu", "block_norm_grad_ring_kernel"), ("block_norm.cu", "block_norm_grad_sums_kernel"), ("quant_i8.cu", "quantize_rows_kernel"),
           ("quant_i8.cu", "quantize_long_rows_kernel"), ("i8_tcgen05.cu", "i8_many_kernel")]


@pytest.mark.parametrize("name,kernel", WAITING)
def test_waits_before_it_reads_and_nothing_read_is_restrict(name, kernel):
    params, body = _kernel(TEXT[name], kernel)
    before = body[:body.index("grid_begin();")]
    if before.strip():
        assert "tcgen05.alloc" in before and "return" not in before
        assert not re.search(r"tma_load|bulk_load|ring_copy|tmem_ld|ld\.global|st\.global", before)
    for p in params.split(","):
        if "__restrict__" in p:
            assert not re.search(r"\bconst\b", p) and _only_written(re.search(r"(\w+)\s*$", p).group(1), body), p
    assert "__restrict__" not in body


def test_the_few_token_product_fetches_only_the_weight_ahead():
    """It takes its tensor memory before it lets the next kernel in; ahead of the wait it asks for the weight and its positions (no kernel
    that is still running writes those: see launch_linear_i8), for the tokens, and reads their scales, behind it."""
    _, body = _kernel(TEXT["i8_tcgen05.cu"], "i8_few_kernel")
    assert body.index("tcgen05.alloc") < body.index("if (!ahead) grid_dependency_wait();") < body.index("grid_launch_dependents();")
    ahead = body.index("if (ahead) grid_dependency_wait();")
    assert body.index("load_w(k0 + i, i)") < ahead < body.index("load_x(k0 + i, i)")
    rounding = body.index("round_rows<BN, X>(p")
    assert "if (ahead) grid_dependency_wait();" in body[body.index("if constexpr (T::RAW)"):rounding]
    out = body.index("if (!*abortp) {")
    assert body.index("grid_dependency_wait();", out) < body.index("p.ws[row]", out) < body.index("p.xs[tok0", out)
    assert not re.search(r"p\.(ws|xs|bias|Y)\b", body[:out])


def test_all_of_their_launches_are_covered():
    """Whatever these files launch as a dependent kernel is named above, or launched through a name that the other tests read."""
    for f in ("block_norm.cu", "quant_i8.cu", "i8_tcgen05.cu"):
        kernels = {re.search(r"(\w+_kernel)\s*\(", TEXT[f][m.end():]).group(1) for m in re.finditer("__global__", TEXT[f])}
        plain = set(re.findall(r"(\w+_kernel)<<<", TEXT[f]))
        assert kernels - plain == {k for g, k in WAITING if g == f} | ({"i8_few_kernel"} if f == "i8_tcgen05.cu" else set())
    assert {k for f, k in LAUNCHED if f == "quant_i8.cu"} == {"quantize_rows_kernel", "quantize_long_rows_kernel"}
