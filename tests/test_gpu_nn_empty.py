"""Matrices without columns are refused with the library's status and message."""
import pytest
import torch

import nn_reference as ref
from paper_2010_13972_amd import gts, nn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ref.DTYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,inputs,outputs", [(4, 0, 5), (4, 3, 0), (4, 0, 0), (0, 0, 5), (0, 3, 0)])
def test_products_without_columns(rows, inputs, outputs, dtype):
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    x, w, dy = (torch.empty(s, dtype=dtype, device="cuda")
                for s in ((rows, inputs), (outputs, inputs), (rows, outputs)))
    for call in (lambda: nn.linear(x, w), lambda: nn.linear_backward(dy, x, w)):
        with pytest.raises(gts.GtsError) as err:
            call()
        assert err.value.status == gts.GTS_EINVAL and "must be >= 1" in str(err.value)


@pytest.mark.parametrize("rows", [0, 4])
def test_norms_without_columns(rows):
    x, w = torch.empty(rows, 0, device="cuda"), torch.empty(0, device="cuda")
    for call in (lambda: nn.norm_residual(x, x, w, w), lambda: nn.norm_residual_backward(x, x, x, x, w, w)):
        with pytest.raises(gts.GtsError) as err:
            call()
        assert err.value.status == gts.GTS_EINVAL
