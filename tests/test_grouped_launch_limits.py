"""Gradients of grouped products whose later launches would not fit a grid: refused before the first launch."""
from test_more_refusals import SIZE, V, grouped_backward


def test_more_biases_than_their_sums_have_threads_for():
    # 32 columns to a block of 256 threads, of which a launch has less than 2^32
    N = 1 << 29
    far = {n: V((k + 1) << 44) for k, n in enumerate(("dC", "off", "db", "ws"))}
    assert grouped_backward(**far, A=None, W=None, pre=None, dA=None, dW=None, act=0, rows=1, groups=1, N=N, K=8, lddc=N, bytes=1 << 40) == SIZE
