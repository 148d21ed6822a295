"""A wait that ran out and an index out of range, noted on one stream: peqa_check_status reports the one and then the other."""
import pytest
import torch

from paper_2305_14152_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("index_first", [False, True])
def test_both_findings_are_reported(index_first):
    w = binding.quantize_rtn(torch.randn((256, 256), device="cuda"), 4, 0)
    X = torch.randn((64, 256), device="cuda").bfloat16()
    table = torch.tensor([[0, 9]], dtype=torch.int32, device="cuda")          # the second page is none of the two
    cache = binding.alloc_kv_cache(2, 16, 1, 64, table)
    rows = torch.randn((1, 1, 64), device="cuda").bfloat16()
    angles, lens = torch.ones((32, 64), device="cuda"), torch.tensor([17], dtype=torch.int32, device="cuda")
    binding.check_status()

    def status():
        with pytest.raises(binding.PeqaError) as err:
            binding.check_status()
        return err.value.status

    calls = [lambda: binding.qlinear_fwd(w, X), lambda: binding.kv_append(cache, rows, rows, rows, angles, lens)]

    binding.selftest_configure(wait_limit_us=1000, starve_forward=True)
    try:
        for call in calls[::-1] if index_first else calls:
            call()
        assert status() == -8                              # PEQA_ERR_DEVICE_TIMEOUT
        assert status() == -10                             # PEQA_ERR_DEVICE_INDEX
        binding.check_status()                             # both read, both cleared
    finally:
        binding.selftest_configure()
    binding.qlinear_fwd(w, X)
    binding.check_status()
