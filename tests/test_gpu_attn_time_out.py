"""The time-out path of the attention over the paged cache: units that never fill must end the kernel through its bounded waits, report
PEQA_ERR_DEVICE_TIMEOUT and leave the context usable.  Nothing traps or spins without a bound: the barriers expect one arrival more than comes, and
waits are limited to a millisecond."""
import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import Case, assert_within


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim,heads,kv_heads,lengths", [(128, 8, 2, [200, 0, 33]), (64, 16, 1, [4000, 17, 0, 900]), (256, 4, 4, [3000] * 9)])
def test_starved_attention_times_out_and_the_next_call_is_correct(dtype, dim, heads, kv_heads, lengths):
    """A CTA for every row, and rows dealt out over all CTAs with the second kernel behind them."""
    case = Case(dim, lengths, heads, kv_heads, dim, 16, dtype)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    ws = binding.alloc_attn_workspace(cache, heads)
    first = binding.attn_decode(cache, q, lens, workspace=ws)
    binding.check_status()
    ref, _, tol, _ = case.attention()
    assert_within(first, ref, tol, "before")
    binding.selftest_configure(wait_limit_us=1000, starve_forward=True)
    try:
        for _ in range(2):
            binding.attn_decode(cache, q, lens, workspace=ws)
        with pytest.raises(binding.PeqaError) as err:
            binding.check_status()
        assert err.value.status == -8                      # PEQA_ERR_DEVICE_TIMEOUT
        binding.check_status()
    finally:
        binding.selftest_configure()
    again = binding.attn_decode(cache, q, lens, workspace=ws)
    binding.check_status()
    assert torch.equal(again, first)
