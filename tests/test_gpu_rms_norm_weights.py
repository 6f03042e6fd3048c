"""fnn_rms_norm where the product of 1 / rms and a weight leaves fp32's range, though the norm and the result do not."""
import pytest
import torch

from net_helpers import TYPES, normal
from test_gpu_rms_norm import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("d", [130, 1024, 5000])
@pytest.mark.parametrize("size,weight", [(1e-5, 1e36), (1e-12, 1e33), (1e18, 1e-24), (1e15, 1e-30), (1.0, 1e-36), (1e-18, 1e34)])
def test_weights_far_from_1(size, weight, d, kind):
    """1 / rms is 1e3 (at most, beside an eps of 1e-6), 1e-18, 1e-15 or 1: times the weight that is above 3.4e38 or below 1.2e-38 for some of these, where digits are lost or all are."""
    dtype = TYPES[kind]
    x, r, w = normal(1, 5, d, std=size, dtype=dtype), normal(2, 5, d, std=size, dtype=dtype), (weight * (1 + normal(3, d, std=0.2)))
    for eps in (1e-6, 1e-30):
        check(x, r, w.to(dtype), eps=eps)
        check(x, None, w, eps=eps)
