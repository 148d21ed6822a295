"""Backward of the gated block's activation for gates so far out that the inner polynomial's slope is beyond binary32."""
import pytest
import torch

from loss_util import assert_within
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_slopes_are_the_limits(act):
    """The activation's slope is 0 far below and 1 far above; the activation itself 0 and the gate."""
    far = torch.tensor([200.0, 1e4, 3e19, 6e19, 1e20, 1e30, 3e38], device="cuda").bfloat16()
    gen = torch.Generator(device="cuda").manual_seed(1)
    T = 37
    gate = torch.cat([far, -far]).repeat(4)[None].repeat(T, 1)
    up = torch.randn(gate.shape, generator=gen, device="cuda").bfloat16()
    dH = (0.1 + 0.4 * torch.rand(gate.shape, generator=gen, device="cuda")).bfloat16()
    Y = torch.stack([gate.unflatten(1, (-1, 8)), up.unflatten(1, (-1, 8))], 2).flatten(1)
    dY = binding.glu_bwd(Y, dH, act).unflatten(1, (-1, 2, 8))
    above = (gate > 0).double()
    # binary32 products of bf16 factors, rounded to bf16; terms good to 2^-18
    for got, want, what in ((dY[:, :, 0].flatten(1), dH.double() * up.double() * above, "gate"),
                            (dY[:, :, 1].flatten(1), dH.double() * gate.double() * above, "up")):
        assert_within(got, want, want.abs() * (2.0 ** -8 + 2.0 ** -17) + 2.0 ** -126, what)
