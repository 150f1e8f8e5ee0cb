"""Layer norm on the GPU of rows whose mean is a million times their spread and more."""
import pytest

from gpu_util import DEV
from test_gpu_z14_layernorm import COLS
from test_gpu_z19_loss_confident import direct
from test_layernorm_far import check_beside, check_far

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [c for c in COLS if c > 1] + [72, 250])
def test_rows_a_million_spreads_from_zero(cols):
    for far in (1e4, 1e6, -4e6):
        check_far(direct, 9, cols, far, dev=DEV)
    check_far(direct, 9, cols, 1e6, spread=0.0, dev=DEV)
    check_far(direct, 2000, cols, 3e5, dev=DEV)


def test_rows_beside_a_far_one_keep_their_bits():
    check_beside(direct, DEV)
