"""Losses and gradients of inputs, and of products, that are not finite: in their rows, and in no others; both kernels, with and without gradient."""
import pytest
import torch

from loss_util import assert_within, inputs, reference
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu

TOKENS = pytest.mark.parametrize("T", [40, 300])
GRAD = pytest.mark.parametrize("grad", [True, False])


def run(X, W, labels, weight, grad):
    loss, dX = binding.head_loss(X, W, labels, weight, need_grad=grad)
    binding.check_status()
    return loss, dX


def check_others(X, W, labels, weight, loss, dX, others):
    want, want_dX, tol, tol_dX = reference(X[others], W, labels[others], weight[others])
    assert_within(loss[others], want, tol, "loss")
    if dX is not None:
        assert_within(dX[others], want_dX, tol_dX, "dX")


@TOKENS
@GRAD
def test_values_stay_in_their_rows(T, grad):
    X, W, labels, weight = inputs(T, 1000, 128, seed=9)
    X[5, 3] = float("nan")
    X[9, 0] = float("inf")
    labels[11] = -1
    X[11] = float("nan")
    loss, dX = run(X, W, labels, weight, grad)
    assert not loss[[5, 9]].isfinite().any() and loss[11] == 0
    if grad:
        assert dX[5].isnan().all() and not dX[9].isfinite().any() and not dX[11].any()
    check_others(X, W, labels, weight, loss, dX, [t for t in range(T) if t not in (5, 9, 11)])


@TOKENS
@GRAD
def test_label_whose_logit_overflows(T, grad):
    """2^100 * 2^30 is beyond binary32, so the label's logit is infinite and all the others are not."""
    X, W, labels, weight = inputs(T, 1000, 128, seed=10)
    X[:, 0] = 0
    W[:, 0] = -1
    labels[labels == 17] = 18
    labels[5] = 17
    X[5, 0], W[17, 0] = 2.0 ** 100, 2.0 ** 30
    loss, dX = run(X, W, labels, weight, grad)
    assert not loss[5].isfinite() and (dX is None or not dX[5].isfinite().any())
    check_others(X, W, labels, weight, loss, dX, [t for t in range(T) if t != 5])


@TOKENS
@GRAD
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_row_of_the_head(T, grad, value):
    """A logit of -inf that is not the label's counts nothing; every other that is not finite makes its token's loss and gradient so."""
    X, W, labels, weight = inputs(T, 1000, 128, seed=11)
    labels[labels == 999] = 998
    labels[4] = 999
    W[999, 3] = value
    logits = torch.where(X[:, 3] == 0, torch.nan, X[:, 3].float() * value)
    # the entry is the last one: without it the vocabulary is a shorter one
    others = ((logits == -torch.inf) & (labels != 999)).nonzero()[:, 0].tolist()
    off = [t for t in range(T) if t not in others]
    assert 4 in off and (value != value or len(others) > T // 4)
    loss, dX = run(X, W, labels, weight, grad)
    assert not loss[off].isfinite().any()
    if grad:
        assert not dX[off].isfinite().any()
    if others:
        want, want_dX, tol, tol_dX = reference(X[others], W[:999], labels[others], weight[others])
        assert_within(loss[others], want, tol, "loss")
        if grad:
            keep = [k for k in range(128) if k != 3]          # 0 * inf in the feature itself
            assert dX[others][:, 3].isnan().all()
            assert_within(dX[others][:, keep], want_dX[:, keep], tol_dX[:, keep], "dX")


@TOKENS
@GRAD
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_vocabulary_of_one(T, grad, value):
    """Nothing but the label: its logit shows in no sum."""
    X, W, labels, weight = inputs(T, 1, 16, seed=12)
    X[:, 0] = 1
    X[3, 0] = value
    loss, dX = run(X, W, labels, weight, grad)
    others = [t for t in range(T) if t != 3]
    assert not loss[3].isfinite() and not loss[others].any()
    if grad:
        assert not dX[3].isfinite().any() and not dX[others].any()
