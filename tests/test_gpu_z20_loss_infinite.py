"""An infinite logit beside large finite ones on the GPU, by every kernel."""
import pytest
import torch

from gpu_util import DEV
from test_gpu_z19_loss_confident import direct
from test_loss_emulated import KERNELS
from test_loss_infinite import check_infinite

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_an_infinite_logit_beside_large_ones(dtype, kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    check_infinite(direct, dtype, DEV)
