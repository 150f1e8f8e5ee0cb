"""The cross entropy's gradients where the vocabulary is long: calls that are accepted or refused by what a slice of it spans, and on the
CPU model of the hardware (tests/emu) several pieces of several slices each."""
import pytest
import torch

import paper_2210_16691_amd as al
from test_loss_emulated import run_gradients
from test_more_refusals import SIZE, V, loss_backward

FAR = {n: V((k + 1) << 44) for k, n in enumerate(("X", "W", "y", "lse", "d", "dX", "dW", "ws"))}


def call(rows, vocab, K, **kw):
    ld = dict(ldx=K, ldw=K, lddx=K, lddw=K)
    need = al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K)
    return loss_backward(**{**FAR, **dict(rows=rows, vocab=vocab, K=K, i=al.BF16, o=al.BF16, bytes=need), **ld, **kw})


# without a GPU a call that passes every check ends at its first launch; with one it would read these addresses
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that are none")


@no_gpu
@pytest.mark.parametrize("rows,vocab,K", [(256, 152064, 8192), (256, 256000, 4608), (64, 131072, 8192), (1, 262144, 5376), (64, 262144, 4096),
                                          (64, 128256, 16384), (512, 128256, 16384), (600, 70000, 16384), (1000, 140000, 16384),
                                          (1, 1 << 22, 8192), (1, 300, 1 << 20)])
def test_vectors_that_span_more_than_2_gib_have_gradients(rows, vocab, K):
    assert call(rows, vocab, K) == al.ERR_LAUNCH
    assert call(rows, vocab, K, dW=None) == al.ERR_LAUNCH
    assert call(rows, vocab, K, dW=None, ldw=2 * K) == al.ERR_LAUNCH        # a pitch of twice the columns


@no_gpu
def test_vectors_too_far_apart_for_a_slice_are_refused():
    # 4096 columns are two slices: 2176 rows of 2^18 numbers are 1.1 GB, of 2^19 2.3 GB
    assert call(8, 4096, 64, dW=None, ldw=1 << 18) == al.ERR_LAUNCH
    assert call(8, 4096, 64, dW=None, ldw=1 << 19) == SIZE
    assert call(8, 4096, 64, dX=None, ldw=1 << 19) == al.ERR_LAUNCH         # dW does not read them


@pytest.mark.parametrize("rows,vocab,K", [(64, 1 << 18, 1 << 12), (600, 70000, 16384), (1, 1 << 22, 8192)])
def test_the_workspace_stays_small(rows, vocab, K):
    # G of a piece (128 MiB), sums of dX of up to 17 slices
    assert al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K) < (129 << 20) + 17 * 4 * rows * K


@pytest.mark.parametrize("dtype,out", [("f16", None), ("bf16", "f32")])
def test_several_pieces_of_several_slices(dtype, out, monkeypatch):
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "8192")
    run_gradients(3, 17000, 16, dtype, out=out, pad=8)            # three pieces of two slices
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "4096")
    run_gradients(2, 34700, 8, dtype, out=out, parts="X")         # eight of two slices and one of one


@pytest.mark.parametrize("dtype,out", [("bf16", None), ("f16", "f32")])
def test_one_piece_of_several_slices(dtype, out):
    run_gradients(2, 8200, 24, dtype, out=out, pad=8)
