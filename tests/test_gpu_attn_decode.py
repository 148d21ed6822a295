"""Attention of one new token per sequence over the paged cache against a plain form in 64 bits.  Whatever may not be read holds no
number: places behind a sequence's end and before its window, pages of no sequence, and the page table behind a sequence's last page."""
import math

import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import Case, assert_within

LENGTHS = [0, 1, 15, 16, 17, 130, 33, 0, 257, 64]


def check(case, what="", **more):
    cache = case.on_gpu()
    out, lse = binding.attn_decode(cache, case.q.cuda(), case.lens(), window=case.window, return_lse=True, **more)
    binding.check_status()
    ref, ref_lse, tol, lse_tol = case.attention(more.get("scale"))
    assert out.dtype == torch.bfloat16 and lse.dtype == torch.float32
    assert_within(out, ref, tol, "out " + what)
    assert_within(lse, ref_lse, lse_tol, "lse " + what)
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 1), (20, 4), (16, 1), (18, 2), (35, 1)])
def test_types_heads_and_lengths(dtype, dim, heads, kv_heads):
    check(Case(dim + heads, LENGTHS, heads, kv_heads, dim, 16, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("page_size", [1, 3, 8, 16, 48, 100, 512])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_pages(dtype, page_size, order):
    check(Case(page_size, LENGTHS, 8, 2, 128, page_size, dtype, order))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("window", [1, 15, 16, 17, 100, 100000])
def test_windows(dtype, window):
    check(Case(window, LENGTHS + [1000], 12, 3, 64, 16, dtype, window=window))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 1, 128), (4, 4, 256), (16, 1, 128), (2, 1, 64)])
@pytest.mark.parametrize("lengths", [[40000], [20001, 3, 0, 7777], [5000] * 5, [16 * 148 * 8], [1] * 700, [0] * 40, [0] * 299 + [9000]])
def test_work_split_over_long_and_many(dtype, heads, kv_heads, dim, lengths):
    if sum(lengths) * kv_heads * dim > 1 << 23:
        lengths = [n // 4 for n in lengths]
    check(Case(len(lengths) + dim, lengths, heads, kv_heads, dim, 16, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_large_and_small_scores(dtype):
    """Scores of hundreds, of which few count; and none at all, an even mean.  Where all but one p are 0 nothing is averaged away."""
    case = Case(5, [300, 1, 64], 8, 2, 128, 16, dtype, spread=6.0)
    check(case, "steep", scale=1.0)
    check(case, "flat", scale=0.0)
    check(case, "turned round", scale=-0.5)


@pytest.mark.gpu
def test_scales_of_any_size():
    """Scales of an 8-bit cache that differ by many powers of ten between tokens: no unit fits all of them."""
    case = Case(6, [200, 77], 8, 2, 128, 16, torch.int8)
    for i, s in enumerate(case.scales):
        t = torch.randint(-12, 12 if i else 1, s.shape, generator=case.gen).double()
        case.scales[i] = (s * 10.0 ** t).float()
    check(case)
    case.scales[1] = torch.zeros_like(case.scales[1])
    out, _ = check(case)
    assert (out == 0).all()
    case.scales[1] += 1e-42                                # subnormal: a value is still what it is
    check(case)


@pytest.mark.gpu
def test_a_head_of_small_numbers_keeps_them():
    """q far below and above 1 with an 8-bit cache."""
    case = Case(7, [100, 30], 4, 2, 64, 16, torch.int8)
    case.q[0] *= 2.0 ** -40
    case.q[1, 0] *= 2.0 ** 100
    check(case, scale=0.125 * 2.0 ** -100)
    case.q[1, 0] *= 2.0 ** -140
    check(case, scale=0.125 * 2.0 ** 40)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_what_is_no_number_stays_with_its_heads(dtype):
    case = Case(8, [50, 60, 70], 8, 4, 64, 16, dtype)
    page, at = case.table[1, 2].item(), 5                  # token 37 of sequence 1
    if dtype == torch.int8:
        case.scales[1][page, 2, at] = math.nan
    else:
        case.kv[1][page, at, 2, 3] = math.nan
    out, lse = binding.attn_decode(case.on_gpu(), case.q.cuda(), case.lens(), return_lse=True)
    ref, ref_lse, tol, lse_tol = case.attention()
    assert torch.equal(out.isnan().cpu(), ref.isnan())
    keep = ~ref.isnan()
    assert_within(out.cpu()[keep], ref[keep], tol[keep], "out")
    assert_within(lse, ref_lse, lse_tol, "lse")


@pytest.mark.gpu
def test_scores_that_are_all_minus_infinity():
    """A key of -inf against a q > 0: a p of 0 where another token has a score, and 0/0 where none has."""
    case = Case(9, [40, 1], 2, 1, 64, 16)
    case.q = case.q.abs() + 0.5
    for b, t in ((0, 7), (1, 0)):
        case.kv[0][case.table[b, t // 16].item(), t % 16] = -math.inf
    out, lse = binding.attn_decode(case.on_gpu(), case.q.cuda(), case.lens(), return_lse=True)
    ref, ref_lse, tol, lse_tol = case.attention()
    assert_within(out[0], ref[0], tol[0], "the others")
    assert_within(lse[0], ref_lse[0], lse_tol[0], "the others' lse")
    assert out[1].isnan().all() and (lse[1] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_strides_and_given_outputs(dtype):
    case = Case(10, LENGTHS, 8, 2, 128, 16, dtype)
    cache, lens = case.on_gpu(), case.lens()
    plain = binding.attn_decode(cache, case.q.cuda(), lens)
    B = len(LENGTHS)
    wide = torch.full((B, 8 + 5, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10] = case.q.cuda()
    given = torch.full((B, 8, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    ws = binding.alloc_attn_workspace(cache, 8)
    got = binding.attn_decode(cache, wide[:, 2:10], lens, out=given, workspace=ws)
    assert got is given and torch.equal(given, plain)
    across = case.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(binding.attn_decode(cache, across, lens), plain)
    # a cache that is a part of a larger pool of several layers
    pool = [torch.zeros((cache.k.shape[0], 3, 2, 16, 128), dtype=dtype, device="cuda") for _ in range(2)]
    for to, x in zip(pool, (cache.k, cache.v)):
        to[:, 1] = x.transpose(1, 2)
    views = [x[:, 1].transpose(1, 2) for x in pool]
    assert torch.equal(binding.attn_decode(binding.KVCache(*views, cache.page_table, cache.k_scales, cache.v_scales),
                                           case.q.cuda(), lens), plain)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_places_beyond_32_bits(dtype):
    """Pages more than 4 GiB into the cache, in elements and bytes."""
    size = 1 if dtype == torch.int8 else 2
    n_pages = (5 << 30) // (size * 16 * 2 * 128) + 9
    shape = (n_pages, 2, 16, 128)
    k, v = (torch.empty(shape, dtype=dtype, device="cuda") for _ in range(2))
    case = Case(11, [70, 20], 4, 2, 128, 16, dtype, spare=0)
    cache = case.on_gpu()
    far = torch.arange(cache.k.shape[0], device="cuda") * 3 + n_pages - 3 * cache.k.shape[0]
    ks = vs = None
    if dtype == torch.int8:
        ks, vs = (torch.empty((n_pages, 2, 16), device="cuda") for _ in range(2))
        ks[far], vs[far] = cache.k_scales, cache.v_scales
    k[far], v[far] = cache.k.transpose(1, 2), cache.v.transpose(1, 2)
    used = (cache.page_table >= 0) & (cache.page_table < cache.k.shape[0])
    table = torch.where(used, far[torch.where(used, cache.page_table, 0).long()].int(), cache.page_table)
    got = binding.attn_decode(binding.KVCache(k.transpose(1, 2), v.transpose(1, 2), table, ks, vs), case.q.cuda(), case.lens())
    binding.check_status()
    assert torch.equal(got, binding.attn_decode(cache, case.q.cuda(), case.lens()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_same_bits_again_and_on_another_stream(dtype):
    case = Case(12, [4000, 1, 900, 0, 77], 16, 2, 128, 16, dtype)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    first = binding.attn_decode(cache, q, lens, return_lse=True)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        second = binding.attn_decode(cache, q, lens, return_lse=True)
    third = binding.attn_decode(cache, q, lens, return_lse=True)
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.gpu
def test_captured_calls_follow_their_inputs():
    """Two captured graphs that share a workspace, replayed in turn with lengths that change between them."""
    case = Case(13, [700, 30, 512, 0], 8, 2, 64, 16)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    ws = binding.alloc_attn_workspace(cache, 8)
    binding.attn_decode(cache, q, lens, workspace=ws)
    graphs, outs = [], []
    for window in (0, 100):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(binding.attn_decode(cache, q, lens, window=window, workspace=ws, return_lse=True))
        graphs.append(g)
    for lengths in ([700, 30, 512, 0], [5, 0, 300, 0], [0, 0, 0, 0], [699, 29, 16, 0]):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        for _ in range(2):
            for g in graphs:
                g.replay()
        for window, got in zip((0, 100), outs):
            want = binding.attn_decode(cache, q, lens, window=window, return_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    binding.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["page too high", "page below 0", "length too high", "length below 0"])
def test_what_is_out_of_range_is_noted_and_left_out(what):
    case = Case(14, [100, 200, 50], 8, 2, 128, 16)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    good = binding.attn_decode(cache, q, lens)
    binding.check_status()
    if what.startswith("page"):
        cache.page_table[1, 3] = cache.k.shape[0] if what.endswith("high") else -1
    else:
        lens[1] = cache.page_table.shape[1] * 16 + 1 if what.endswith("high") else -5
    got = binding.attn_decode(cache, q, lens)
    with pytest.raises(binding.PeqaError) as err:
        binding.check_status()
    assert err.value.status == -10
    if what.startswith("page"):                            # (another length deals the work out in another way)
        assert torch.equal(got[0], good[0]) and torch.equal(got[2], good[2])
    else:
        ref, _, tol, _ = case.attention()
        for b in (0, 2):
            assert_within(got[b], ref[b], tol[b], "the others")
    binding.check_status()                                 # read once, cleared


@pytest.mark.gpu
def test_refusals():
    case = Case(15, [100, 200], 8, 2, 128, 16)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    attend = binding.attn_decode
    for bad_q in (q.float(), q[:, :, :64], q[:1], q.reshape(2, -1), q.transpose(1, 2).contiguous().transpose(1, 2), case.q):
        with pytest.raises(ValueError):
            attend(cache, bad_q, lens)
    for bad_lens in (lens.long(), lens[:1], lens.cpu()):
        with pytest.raises(ValueError):
            attend(cache, q, bad_lens)
    with pytest.raises(ValueError):
        attend(cache, q, lens, out=torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        attend(cache, q, lens, window=1 << 40)

    def status(*args, **kw):
        with pytest.raises(binding.PeqaError) as err:
            attend(*args, **kw)
        return err.value.status

    odd = torch.zeros((2, 7, 128), dtype=torch.bfloat16, device="cuda")
    assert status(cache, odd, lens) == -3                  # heads are no multiple of the cache's
    assert status(cache, q, lens, window=-1) == -3
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    assert status(cache, q, lens, workspace=small) == -5
    ws = binding.alloc_attn_workspace(cache, 8)
    assert status(cache, q, lens, workspace=torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:]) == -4
    shifted = torch.zeros(2 * 8 * 128 + 8, dtype=torch.bfloat16, device="cuda")[1:2 * 8 * 128 + 1].view(2, 8, 128)
    assert status(cache, shifted, lens) == -4
    with pytest.raises(ValueError):
        attend(binding.KVCache(cache.k, cache.v[:, :8], cache.page_table), q, lens)
    with pytest.raises(ValueError):
        attend(binding.KVCache(cache.k, cache.v.contiguous(), cache.page_table), q, lens)      # other strides than k's
    with pytest.raises(ValueError):
        attend(binding.KVCache(cache.k, cache.v, cache.page_table.long()), q, lens)
    same = lambda x: x[:1].expand(4, *x.shape[1:])         # four pages in one place
    assert status(binding.KVCache(same(cache.k), same(cache.v), cache.page_table), q, lens) == -3
    binding.check_status()
    attend(cache, q, lens)


@pytest.mark.gpu
def test_outputs_over_the_queries_are_refused():
    """Several warps read a row of queries, the last perhaps when the first has written its outputs."""
    case = Case(16, [100, 200], 8, 2, 128, 16)
    cache, lens = case.on_gpu(), case.lens()
    pool = torch.zeros((5, 8, 128), dtype=torch.bfloat16, device="cuda")
    pool[1:3] = case.q.cuda()
    q = pool[1:3]
    for out in (q, pool[0:2], pool[2:4]):
        with pytest.raises(ValueError, match="out: expected memory apart from q"):
            binding.attn_decode(cache, q, lens, out=out)
    assert torch.equal(binding.attn_decode(cache, q, lens, out=pool[3:5]), binding.attn_decode(cache, case.q.cuda(), lens))
    assert torch.equal(q, case.q.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [5, 33, 1000, 2 ** 31 - 1])
def test_windows_where_the_work_is_dealt_out(dtype, dim, window):
    """More rows than CTAs; first and last tiles are cut by the window, the end or both."""
    lengths = [1500, 0, 1, 999, 1001] + [16 * i + i % 17 for i in range(60)]
    check(Case(dim + window % 64, lengths, 6, 3, dim, 16 if dim != 256 else 48, dtype, window=window))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,n", [(8, 2, 74), (8, 2, 75), (4, 1, 37), (4, 1, 36)])
def test_about_as_many_rows_as_ctas(heads, kv_heads, n):
    lengths = [(37 * i) % 300 for i in range(n)]
    check(Case(n, lengths, heads, kv_heads, 64, 16))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("window", [0, 9])
def test_many_rows_of_few_tokens(dtype, dim, order, window):
    """Last tiles of 1 to 16 tokens, and cut on both sides by the window; what lies behind is no number."""
    check(Case(dim + window, [1 + (7 * i) % 41 for i in range(100)] + [0, 8, 16, 24], 6, 3, dim, 16, dtype, order, window=window))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("longest", [495, 496, 497, 513])
def test_few_rows_of_about_32_tiles(dtype, longest):
    check(Case(longest, [longest, 300, 0, 17], 4, 2, 64, 16, dtype))


@pytest.mark.gpu
def test_more_sequences_than_a_list_of_the_empty_ones_holds():
    lengths = [(i % 5 - 2) * (i % 7 == 3) * (i % 5 > 2) for i in range(5200)]
    out, lse = check(Case(17, lengths, 2, 1, 64, 16))
    none = torch.tensor(lengths, device="cuda") == 0
    assert (out[none] == 0).all() and (lse[none] == -math.inf).all() and (lse[~none] > -math.inf).all()
