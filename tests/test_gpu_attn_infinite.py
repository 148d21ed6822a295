"""Infinities among the cached values of a bf16 cache: sum_t p_t v_t is that infinity in its channel, whatever p is made of (no number where both
signs meet), and the other channels and heads are what they are without it."""
import math

import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import Case, assert_within


def _check(case, spots):
    """spots: (sequence, token, key-value head, channel, value)"""
    for b, t, h, c, x in spots:
        case.kv[1][case.table[b, t // case.page].item(), t % case.page, h, c] = x
    out, lse = binding.attn_decode(case.on_gpu(), case.q.cuda(), case.lens(), window=case.window, return_lse=True)
    binding.check_status()
    ref, ref_lse, tol, lse_tol = case.attention()
    assert torch.equal(out.isnan().cpu(), ref.isnan())
    assert (ref.isinf().sum() > 0) and torch.equal(out.double().cpu()[ref.isinf()], ref[ref.isinf()])
    keep = ref.isfinite()
    assert_within(out.cpu()[keep], ref[keep], tol[keep], "out")
    assert_within(lse, ref_lse, lse_tol, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 2), (8, 1), (16, 1), (20, 1)])
@pytest.mark.parametrize("page_size", [16, 24])
def test_one_token_and_a_few(dim, heads, kv_heads, page_size):
    """A lone token's p is 1, which bf16 holds exactly; of two tokens with one key p is 1/2 each."""
    case = Case(dim + heads, [1, 2, 40, 17], heads, kv_heads, dim, page_size)
    page = case.table[1, 0].item()
    case.kv[0][page, 1] = case.kv[0][page, 0]
    h = kv_heads - 1
    _check(case, [(0, 0, 0, 0, math.inf), (0, 0, h, dim - 1, -math.inf), (1, 0, h, 5, math.inf), (1, 1, 0, 6, -math.inf), (1, 0, 0, 9, math.inf),
                  (1, 1, 0, 9, -math.inf), (2, 33, 0, 3, math.inf), (2, 2, h, 8, -math.inf), (3, 16, 0, 1, math.inf), (3, 0, 0, 1, math.inf)])


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 1), (16, 1)])
@pytest.mark.parametrize("lengths", [[330, 50, 300], [30000, 9], [16 * (1 + i % 5) for i in range(200)]])
def test_parts_of_rows(heads, kv_heads, lengths):
    """Rows that several warps, or several CTAs, have parts of: an odd number of parts and an even one, the infinity in the first and in the last.
    (Flat scores: no p of a row is lost beside another.)"""
    case = Case(len(lengths), lengths, heads, kv_heads, 64, 16)
    case.q *= 0.25
    _check(case, [(0, 1, 0, 0, math.inf), (0, lengths[0] - 1, 0, 1, -math.inf), (0, lengths[0] // 2, 0, 2, math.inf), (1, 0, kv_heads - 1, 63, math.inf),
                  (len(lengths) - 1, 7, 0, 33, -math.inf), (len(lengths) - 1, 8, 0, 34, math.inf)])


@pytest.mark.gpu
def test_what_is_not_seen_may_be_infinite():
    """Before a window, behind the end and in other pages."""
    case = Case(31, [50, 70, 3], 8, 2, 128, 16, window=20)
    for x in case.kv:
        x[~case.seen] = math.inf
    out = binding.attn_decode(case.on_gpu(), case.q.cuda(), case.lens(), window=20)
    ref, _, tol, _ = case.attention()
    assert_within(out, ref, tol, "out")
