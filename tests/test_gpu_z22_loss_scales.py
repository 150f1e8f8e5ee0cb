"""Gradients of the cross entropy in fp16 on the GPU for losses that weigh next to nothing or enormously."""
import pytest

from gpu_util import DEV
from test_gpu_z19_loss_confident import direct
from test_loss_scales import check_scale

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-33, 1e-30, 1.0, 1e30, 2e36])
def test_losses_of_every_weight(size):
    check_scale(direct, size, dev=DEV)
    check_scale(direct, size, rows=1200, vocab=3000, K=136, dev=DEV)
