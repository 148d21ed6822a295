"""What the binding refuses of a cache and of the rows of an append: by shapes, strides and addresses alone, so without a GPU too."""
import pytest
import torch

from paper_2305_14152_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def _cache(pages=3, page_size=16, kv_heads=2, dim=64, dtype=torch.int8, device="cpu"):
    return binding.alloc_kv_cache(pages, page_size, kv_heads, dim, torch.zeros((1, 2), dtype=torch.int32, device=device), dtype)


def _calls(cache):
    device = cache.k.device
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device=device)
    lens = torch.ones(1, dtype=torch.int32, device=device)
    yield lambda: binding.attn_decode(cache, q, lens)
    yield lambda: binding.kv_append(cache, q, q[:, :2], q[:, 2:], torch.zeros((9, 64), device=device), lens)


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
@pytest.mark.parametrize("name", ["k_scales", "v_scales"])
@pytest.mark.parametrize("shape", [(3, 16, 2), (3 * 16 * 2,), (3, 2, 4, 4), (3, 2, 15), (2, 3, 16)])
def test_scales_in_another_shape(device, name, shape):
    """[n_pages, page_size, n_kv_heads] is the order of codes whose tokens keep their heads together: as many values, other tokens'."""
    cache = _cache(device=device)
    setattr(cache, name, torch.ones(shape, device=device))
    for call in _calls(cache):
        with pytest.raises(ValueError, match=rf"cache.{name}: expected \[n_pages, n_kv_heads, page_size\]"):
            call()


@pytest.mark.gpu
def test_scales_of_the_right_shape_are_taken():
    cache = _cache(device="cuda")
    for call in _calls(cache):
        call()
    cache.k_scales = torch.ones((3, 16, 2), device="cuda").transpose(1, 2)     # the shape, in other strides
    for call in _calls(cache):
        with pytest.raises(ValueError, match="k_scales: expected a contiguous CUDA tensor"):
            call()
    binding.check_status()
