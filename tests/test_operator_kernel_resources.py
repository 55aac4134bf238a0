"""Compile-time guard for the kernels of the operators: their registers decide how many waves hide each other's reads, and a
spill in a loop costs more than the wave it saves."""
from test_kernel_resources import resource_usage


def without_spills(source, allowed=()):
    kernels = resource_usage(source)
    bad = {k: v for k, v in kernels.items() if v["scratch"] and not any(a in k for a in allowed)}
    assert kernels and not bad, bad
    return kernels


def waves(kernels, part):
    found = [v["waves"] for k, v in kernels.items() if part in k]
    assert found, part
    return min(found)


def test_norm_kernels():
    """Rows of 8193 to 16384 columns from codes use what registers sixteen waves leave each other, and a few words of scratch
    before their loop."""
    kernels = without_spills("qa_norm.hip", ("rms_norm_grad_kernelILi0ELi1024ELi2ELb1E", "rms_norm_grad_kernelILi1ELi1024ELi2ELb1E"))
    assert all(v["scratch"] <= 32 for v in kernels.values())
    assert waves(kernels, "15rms_norm_kernel") >= 5 and waves(kernels, "rms_norm_grad_kernel") >= 3


def test_row_kernels():
    assert waves(without_spills("qa_rows.hip"), "rows_") == 8


def test_token_kernels():
    kernels = without_spills("qa_token.hip")
    for part, least in (("token_wide_kernel", 4), ("token_narrow_kernel", 5), ("token_grad_kernel", 3)):
        assert waves(kernels, part) >= least, part
    # four work-groups of a wide row per compute unit
    assert all(v["lds"] <= 40 * 1024 for k, v in kernels.items() if "token_wide" in k)


def test_weight_gradient_kernels():
    """Two waves per SIMD: the tile of 256 x 256 is eight waves with 128 sums each."""
    kernels = without_spills("qa_weight_grad.hip")
    assert waves(kernels, "weight_grad_kernel") >= 2
    assert all(v["lds"] <= 160 * 1024 for v in kernels.values())
