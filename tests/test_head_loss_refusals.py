"""What peqa_head_loss refuses before it touches a device, and the size of its workspace."""
import ctypes

import pytest
import torch

from paper_2305_14152_b200 import binding, build

NULL, SHAPE, ALIGN, WORKSPACE, LARGE = -1, -3, -4, -5, -9


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(4096)
    yield (ctypes.addressof(buf) + 255) & ~255
    del buf


def call(L, p, X=1, W=1, labels=1, weight=0, T=4, V=100, K=64, loss=1, dX=1):
    at = lambda v: p if v == 1 else v
    return L.peqa_head_loss(at(X), at(W), at(labels), at(weight), T, V, K, at(loss), at(dX), p, 1 << 40, 0)


def test_refusals(L, p):
    for name in ("X", "W", "labels", "loss"):
        assert call(L, p, **{name: 0}) == NULL, name
        assert call(L, p, **{name: p + 8}) == ALIGN, name
    assert call(L, p, dX=p + 2) == ALIGN and call(L, p, weight=p + 4) == ALIGN
    for sizes in ({"T": 0}, {"T": -1}, {"V": 0}, {"V": -5}, {"K": 0}, {"K": 4}, {"K": 100}, {"K": -8}):
        assert call(L, p, **sizes) == SHAPE, sizes
    for sizes in ({"T": (1 << 24) + 1}, {"V": (1 << 24) + 1}, {"K": (1 << 20) + 8}):
        assert call(L, p, **sizes) == LARGE, sizes


def test_workspace(L):
    of = lambda T, V, K, grad: L.peqa_head_loss_workspace_bytes(T, V, K, grad)
    assert of(0, 100, 64, 1) == of(1, 0, 64, 1) == of(1, 100, 60, 1) == of(1 << 25, 100, 64, 1) == 0
    # never as much as the logits in binary32 where these are large
    for T, V, K in ((4096, 128000, 4096), (8192, 50257, 8192), (65536, 32000, 4096)):
        assert 0 < of(T, V, K, 0) < of(T, V, K, 1) < 4 * T * V
    # beside what grows with the tokens (their rows), bounded
    assert of(1 << 20, 32000, 4096, 1) < (1 << 20) * (2 * 4096 + 64) + (1 << 30)


def test_binding_refuses_what_does_not_belong_together():
    X = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous CUDA tensor"):
        binding.head_loss(X, X, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(binding.PeqaError):
        binding.alloc_head_loss_workspace(X[:, :60], torch.zeros(9, 60))
