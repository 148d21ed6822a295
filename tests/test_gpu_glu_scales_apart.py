"""Forward of a gated block whose groups' scales are far apart within a row: a group far below its row's largest keeps its bits."""
import pytest
import torch

from glu_util import block, forward, weights
from loss_util import assert_within
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("apart", [12, 17, 23])
@pytest.mark.parametrize("T", [30, 600])
def test_groups_far_below_the_rows_largest(T, apart, group, bits):
    """Channels of the large groups are 0, so every sum is made of the small ones, which count in full: two half steps of binary16 a product, as
    everywhere, and no term that follows the row's largest scale."""
    F, K = 40, 512
    w, _, codes = block(F, K, bits, group, seed=apart + group)
    w.scales[:, 1::2] *= 2.0 ** -apart
    small = (torch.arange(K, device="cuda") // group % 2 == 1)
    X = (torch.randn((T, K), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda") * small).bfloat16()
    W = weights(codes, w.zeros, w.scales) * small
    H, Y = binding.qglu_fwd(w, X)
    binding.check_status()
    want, want_Y, tol, tol_Y = forward(X, W, "silu", True)
    assert_within(Y, want_Y, tol_Y, "Y")
    assert_within(H, want, tol, "H")


@pytest.mark.parametrize("T", [30, 600])
def test_largest_codes_at_the_largest_scale(T):
    """(Q - z) s of the largest code and the smallest zero-point, and the other way round, stay within binary16."""
    F, K, g = 24, 256, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    codes = torch.full((2 * F, K), 15, dtype=torch.uint8, device="cuda")
    codes[1::2] = 0
    zeros = torch.where(codes[:, ::g] == 0, 15, 0).to(torch.uint8)
    scales = torch.full((2 * F, K // g), 1.9999 * K ** -1.0 / 15, device="cuda")
    w = binding.QWeight(4, 2 * F, K, g, binding.pack(codes, 4), zeros, scales)
    X = (16 * torch.rand((T, K), generator=gen, device="cuda")).bfloat16()
    H, Y = binding.qglu_fwd(w, X)
    want, want_Y, tol, tol_Y = forward(X, weights(codes, zeros, scales), "silu", True)
    assert_within(Y, want_Y, tol_Y, "Y")
    assert_within(H, want, tol, "H")
