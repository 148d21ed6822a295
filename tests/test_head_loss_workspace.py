"""One workspace of the loss serves every batch up to the tokens that it was made for."""
import random

import pytest
import torch

from loss_util import assert_within, inputs, reference
from paper_2305_14152_b200 import binding, build


def test_size_grows_with_the_tokens():
    build.build()
    of = binding.lib().peqa_head_loss_workspace_bytes
    rng = random.Random(1)
    sizes = [(32000, 4096), (50257, 4096), (131072, 4096), (20000, 256), (1, 8), (300, 1 << 18), (1 << 20, 64)]
    sizes += [(int(2 ** rng.uniform(0, 18)), 8 * int(2 ** rng.uniform(0, 11))) for _ in range(20)]
    lengths = [1, 2, 256, 257] + list(range(512, 9000, 253)) + [20000, 65536, 65537, 200000]
    for V, K in sizes:
        for grad in (0, 1):
            bytes_ = [of(T, V, K, grad) for T in lengths]
            assert all(0 < a <= b for a, b in zip(bytes_, bytes_[1:])), (V, K, grad)


@pytest.mark.gpu
@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("V,K,longest,shorter", [(50257, 64, 2017, (1537, 150, 1)), (20000, 256, 5057, (4609, 257, 256)), (131072, 64, 257, (256, 31, 1))])
def test_shorter_batches(V, K, longest, shorter, grad):
    X, W, labels, weight = inputs(longest, V, K, seed=V)
    ws = binding.alloc_head_loss_workspace(X, W, grad)
    for T in (longest, *shorter):
        part = X[:T].contiguous(), W, labels[:T].clone(), weight[:T].clone()
        loss, dX = binding.head_loss(*part, need_grad=grad, workspace=ws)
        binding.check_status()
        want, want_dX, tol, tol_dX = reference(*part)
        assert_within(loss, want, tol, "loss")
        if grad:
            assert_within(dX, want_dX, tol_dX, "dX")
