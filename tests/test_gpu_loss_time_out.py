"""The time-out path of the kernels of the loss and of the gated block: stages that never fill must end them through their bounded
waits, report PEQA_ERR_DEVICE_TIMEOUT and leave the context usable.  Nothing traps or spins without a bound: one byte more is announced than the copies
deliver, and waits are limited to a millisecond."""
import pytest
import torch

from glu_util import block
from loss_util import inputs
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu


def starved(call):
    first = [t.clone() for t in call() if t is not None]
    binding.check_status()
    binding.selftest_configure(wait_limit_us=1000, starve_forward=True)
    try:
        call()
        with pytest.raises(binding.PeqaError) as err:
            binding.check_status()
        assert err.value.status == -8                      # PEQA_ERR_DEVICE_TIMEOUT
        binding.check_status()
    finally:
        binding.selftest_configure()
    again = [t for t in call() if t is not None]
    binding.check_status()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("T,V,K", [(40, 3000, 256), (700, 3000, 256), (3000, 30000, 128)])
@pytest.mark.parametrize("grad", [True, False])
def test_loss(T, V, K, grad):
    X, W, labels, weight = inputs(T, V, K, seed=1)
    starved(lambda: binding.head_loss(X, W, labels, weight, need_grad=grad))


@pytest.mark.parametrize("T", [2000, 4096])
@pytest.mark.parametrize("group", [0, 64])
def test_gated_block(T, group):
    w, _, _ = block(4096, 1024, 4, group, seed=2)
    X = torch.randn((T, 1024), device="cuda").bfloat16()
    starved(lambda: binding.qglu_fwd(w, X))


@pytest.mark.parametrize("group", [0, 64])
def test_wide_gated_block_of_few_tokens(group):
    """Two launches side by side."""
    w, _, _ = block(10240, 1024, 4, group, seed=3)
    X = torch.randn((33, 1024), device="cuda").bfloat16()
    starved(lambda: binding.qglu_fwd(w, X))
