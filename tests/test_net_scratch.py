"""The operators' kernels keep their sums in registers: scratch memory would put them into the inner loops' way.  The gradient of attention's second
pass at more than 96 elements, and tiles through registers at as many, may spill a few."""
import re

import pytest

from test_kernel_scratch import scratch_bytes


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    return scratch_bytes(tmp_path_factory.mktemp("notes"))


@pytest.mark.parametrize("kernel,at_least", [
    (r"gemm_kernelI.*Lb1EE", 12), (r"few_rows_kernelI", 9), (r"layer_norm_kernelI", 30), (r"slope_kernelI", 3), (r"attention_kernelI.*Lb1EE", 8),
    (r"attention_few_kernelI", 16), (r"attention_dq_kernelI.*Lb1EE", 8), (r"attention_dkv_kernelILi[12]ELi[123]E", 12)])
def test_no_scratch_memory(scratch, kernel, at_least):
    found = {k: v for k, v in scratch.items() if re.search(r"\d" + kernel, k)}
    assert len(found) >= at_least
    assert not {k: v for k, v in found.items() if v}
