"""Calls of the cross entropy whose later launches would not fit a grid, or whose factor leaves fp32: refused before the first
launch."""

import paper_2210_16691_amd as al
from test_loss_far import FAR
from test_more_refusals import SIZE, UNSUPPORTED, V, loss, loss_backward

WHERE = {n: FAR[n] for n in ("X", "W", "y", "lse", "ws")}


def test_more_rows_than_the_merge_has_threads_for():
    # 32 rows to a block of 1024 threads, of which a launch has less than 2^32
    assert loss(**WHERE, out=V(9 << 44), rows=1 << 27, vocab=8, K=8, ldx=8, ldw=8, bytes=1 << 40) == SIZE


def test_more_results_than_their_rounding_has_threads_for():
    kw = dict(FAR, rows=1 << 22, vocab=5000, K=8192, ldx=8192, ldw=8192, lddx=8192, bytes=1 << 41, dW=None)
    assert loss_backward(**kw, i=al.BF16, o=al.BF16) == SIZE


def test_a_factor_that_leaves_fp32_in_exponents_of_2():
    # 2.4e38 log2(e) is infinite in fp32, and 0 times it makes a logit of 0 NaN
    for f, where in ((loss, WHERE), (loss_backward, FAR)):
        assert f(**where, alpha=2.4e38) == UNSUPPORTED
        assert f(**where, alpha=1e38, bytes=64) == SIZE          # (a factor that is taken, a workspace that is not)
