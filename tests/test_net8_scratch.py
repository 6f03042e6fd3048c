"""The kernels of matrices in 8 bits keep their sums in registers.  Tiles whose operands go through registers may spill a few, for fp32 results, and so may the gradient of the norm of rows that
take a workgroup of 1024 threads each."""
import re

import pytest

from test_kernel_scratch import scratch_bytes


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    return scratch_bytes(tmp_path_factory.mktemp("notes"))


@pytest.mark.parametrize("kernel,at_least", [
    (r"gemm_e4m3_kernelI.*Lb1EE", 10), (r"gemm_small_e4m3_kernelI", 6), (r"few_rows_e4m3_kernelI", 6), (r"gradient_small_e4m3_kernelI", 3), (r"copy_codes_kernelE", 1),
    (r"quantize_rows_kernelI", 3), (r"quantize_tile_kernelI", 6), (r"gradient_operands_kernelI", 3), (r"rms_norm_kernelI", 30), (r"rms_norm_backward_kernelILi[012]ELi[012]ELi(64|256)E", 15)])
def test_no_scratch_memory(scratch, kernel, at_least):
    found = {k: v for k, v in scratch.items() if re.search(r"\d" + kernel, k)}
    assert len(found) >= at_least, sorted(found)
    assert not {k: v for k, v in found.items() if v}
