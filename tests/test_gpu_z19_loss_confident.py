"""The loss of rows that are predicted well on the GPU, by every kernel."""
import pytest
import torch

from gpu_util import DEV
from test_loss_confident import check_confident
from test_loss_emulated import KERNELS

pytestmark = pytest.mark.gpu


def direct(fn, *args, **kw):
    fn(*args, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("behind", [None, 3, -3])
@pytest.mark.parametrize("dtype,alpha", [(torch.float16, 1.0), (torch.bfloat16, 1.0), (torch.float16, 0.25)])
def test_the_loss_of_confident_rows(dtype, alpha, behind, kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    check_confident(direct, dtype, behind, alpha, DEV)
