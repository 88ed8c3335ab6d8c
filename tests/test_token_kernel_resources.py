"""Resources the compiler gave the token kernels: a register spilled inside an attention loop is a load that waits for all requests before it (the loop over a
long cache took twice the time), and results do not show it."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("kernel", ["quant_rows_kernel", "quant_matvec_kernel", "quant_matmul_kernel", "quant_finish_kernel", "cache_write_kernel", "cache_read_kernel", "logprobs_kernelI\\w+Lb0E",
                                    "logprobs_join_kernel", "attention_join_kernel", "attention_kernelILi[123]", "attention_tile_kernelILi[123]"])
def test_no_vector_register_is_spilled(kernels, kernel):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.search(r"\d" + kernel, k)}
    assert found, kernel
    assert not {k: v for k, v in found.items() if v["vgpr_spill_count"] or v["private_segment_fixed_size"]}


@pytest.mark.parametrize("kernel,most", [("attention_kernelILi1E", 168), ("attention_kernelILi2E", 256), ("attention_tile_kernelILi[12]E", 256), ("logprobs_kernelI", 64),
                                         ("quant_matmul_kernelI\\w+Li4ELi2ELi2E", 256)])
def test_units_hold_the_wavefronts_that_were_planned(kernels, kernel, most):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.search(r"\d" + kernel, k)}
    assert found and not {k: v["vgpr_count"] for k, v in found.items() if v["vgpr_count"] > most}


@pytest.mark.parametrize("kernel,most", [("logprobs_kernelI\\w+Lb1E", 4), ("attention_kernelILi4E", 6), ("attention_tile_kernelILi4E", 21)])
def test_few_registers_are_spilled_where_some_are(kernels, kernel, most):  # noqa: F811
    """Best tokens at eight wavefronts a unit, and heads beyond 192: what they spill is known, and small."""
    found = {k: v for k, v in kernels.items() if re.search(r"\d" + kernel, k)}
    assert found and not {k: v["vgpr_spill_count"] for k, v in found.items() if v["vgpr_spill_count"] > most}
