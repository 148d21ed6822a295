"""The paged cache in layouts and sizes that other tests do not reach: pages, tokens and heads in every order, page tables wider than the sequences, runs of an
8-bit append in other layouts and without queries, and an append more than 4 GiB into the cache."""
import itertools

import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import Case, assert_within
from test_gpu_kv_append import Batch
from test_gpu_kv_append import check as check_append

ORDERS = ["".join(o) for o in itertools.permutations("pth")]            # of pages, tokens and heads, outermost first


def lay_out(x, order):
    """[n_pages, page_size, n_kv_heads, head_dim] on the GPU, its dimensions in this order in memory."""
    to = ["pth".index(c) for c in order]
    return x.permute(*to, 3).contiguous().cuda().permute(*[to.index(i) for i in range(3)], 3)


def _attend(case, cache):
    out, lse = binding.attn_decode(cache, case.q.cuda(), case.lens(), window=case.window, return_lse=True)
    binding.check_status()
    ref, ref_lse, tol, lse_tol = case.attention()
    assert_within(out, ref, tol, "out")
    assert_within(lse, ref_lse, lse_tol, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dim,page_size", [(64, 16), (128, 32), (256, 16), (128, 5)])
def test_attention_in_any_order(dtype, order, dim, page_size):
    """Through tensor copies where a tile lies in one page, else token by token."""
    case = Case(dim + page_size, [0, 1, 33, 16, 250, 77], 12, 3, dim, page_size, dtype)
    cache = case.on_gpu()
    views = [lay_out(x, order) for x in case.kv]
    assert [views[0].stride(i) for i in ("pth".index(c) for c in order)] == sorted(views[0].stride()[:3], reverse=True)
    _attend(case, binding.KVCache(*views, cache.page_table, cache.k_scales, cache.v_scales))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("page_size", [1, 16, 24])
def test_appending_in_any_order(dtype, order, page_size):
    batch = Batch(page_size, [37, 90, 5, 12, 0], [37, 33, 1, 0, 0], 8, 3, 64, page_size, dtype, before=1, behind=2)
    _, want = check_append(batch)
    cache = batch.on_gpu()
    cache.k, cache.v = (lay_out(x, order) for x in batch.cache)
    q, k, v, cos_sin, lens, starts = batch.args()
    binding.kv_append(cache, q, k, v, cos_sin, lens, starts)
    binding.check_status()
    for a, b in ((cache.k, want.k), (cache.v, want.v)) + (((cache.k_scales, want.k_scales), (cache.v_scales, want.v_scales)) if dtype == torch.int8 else ()):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("seqs,heads,kv_heads,dim", [(1, 8, 2, 128), (5, 8, 8, 64), (40, 16, 4, 128), (200, 4, 2, 64)])
@pytest.mark.parametrize("window", [0, 21])
def test_tables_wider_than_the_sequences(dtype, order, seqs, heads, kv_heads, dim, window):
    """As a captured step has them: room for thousands of tokens, of which few are there; behind a sequence's last page the table holds numbers of no page."""
    case = Case(seqs + dim, [(29 * i + 130) % 140 for i in range(seqs)], heads, kv_heads, dim, 16, dtype, order, width=400, window=window)
    _attend(case, case.on_gpu())


# 8-bit calls of more than 56 items an SM, 16 heads of 128 (32 of 64) an item, are taken in runs
@pytest.mark.gpu
@pytest.mark.parametrize("order,page_size", [("tokens", 3), ("tokens", 48), ("heads", 48), ("tokens", 16)])
@pytest.mark.parametrize("dim,tokens,heads,kv_heads", [(128, 1800, 64, 8), (64, 2900, 64, 16), (256, 1400, 40, 8)])
def test_runs_in_other_layouts(order, page_size, dim, tokens, heads, kv_heads):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    batch = Batch(dim + page_size, [tokens + 99, 9, 0, 401], [tokens, 1, 0, 400], heads, kv_heads, dim, page_size, torch.int8, order, rotary=dim // 2, before=2, behind=3)
    assert batch.q.shape[0] * -(-(heads + 2 * kv_heads) // (2048 // dim)) > 56 * sms
    check_append(batch)


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_runs_of_keys_and_values_alone(order):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    batch = Batch(41, [900, 40, 300], [800, 0, 299], 1, 70, 128, 24, torch.int8, order, behind=4)
    assert batch.q.shape[0] * -(-140 // 16) > 56 * sms
    _, want = check_append(batch)
    cache = batch.on_gpu()
    _, k, v, cos_sin, lens, starts = batch.args()
    assert binding.kv_append(cache, None, k, v, cos_sin, lens, starts) is None
    binding.check_status()
    for a, b in ((cache.k, want.k), (cache.v, want.v), (cache.k_scales, want.k_scales), (cache.v_scales, want.v_scales)):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tokens", [(torch.bfloat16, 70), (torch.int8, 70), (torch.int8, 2100)])
def test_appending_beyond_32_bits(dtype, tokens):
    """Pages more than 4 GiB into the cache, in elements and bytes; one item a CTA, and runs (2100 tokens)."""
    size, kv_heads = 1 if dtype == torch.int8 else 2, 32
    n_pages = (5 << 30) // (size * 16 * kv_heads * 128) + 9
    batch = Batch(42, [tokens + 5, 20], [tokens, 20], 8, kv_heads, 128, 16, dtype)
    near = batch.on_gpu()
    args = batch.args()
    want = binding.kv_append(near, *args[:5], args[5])
    k, v = (torch.zeros((n_pages, kv_heads, 16, 128), dtype=dtype, device="cuda") for _ in range(2))
    far = torch.arange(near.k.shape[0], device="cuda") * 3 + n_pages - 3 * near.k.shape[0]
    ks = vs = None
    if dtype == torch.int8:
        ks, vs = (torch.zeros((n_pages, kv_heads, 16), device="cuda") for _ in range(2))
    used = (near.page_table >= 0) & (near.page_table < near.k.shape[0])
    table = torch.where(used, far[torch.where(used, near.page_table, 0).long()].int(), near.page_table)
    got = binding.kv_append(binding.KVCache(k.transpose(1, 2), v.transpose(1, 2), table, ks, vs), *args[:5], args[5])
    binding.check_status()
    assert torch.equal(got, want)
    fresh = batch.on_gpu()                                     # where nothing was written the far cache has zeros
    for cache, x, near_x, old in ((k, "k", near.k, fresh.k), (v, "v", near.v, fresh.v)):
        at = cache[far].transpose(1, 2)
        touched = torch.zeros(near_x.shape[:2], dtype=torch.bool, device="cuda")
        _, page, place = batch.expected()
        touched[page.cuda(), place.cuda()] = True
        assert torch.equal(at[touched], near_x[touched]) and not at[~touched].any(), x
        assert int((cache != 0).any(-1).any(-1).any(-1).sum()) == int(touched.any(1).sum()), x   # no other page
    if dtype == torch.int8:
        for far_s, near_s in ((ks, near.k_scales), (vs, near.v_scales)):
            assert torch.equal(far_s[far].transpose(1, 2)[touched], near_s.transpose(1, 2)[touched])
