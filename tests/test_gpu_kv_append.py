"""New keys and values into the paged cache, and the rotation, against plain forms: the rotated values in 64 bits, the codes of
an 8-bit cache bit for bit in binary32.  Everything that no token has its place in stays as it was."""
import math

import numpy as np
import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import BF16_HALF_STEP, H, angles, assert_within, page_table, places, quantized, rotated32


class Batch:
    """counts new tokens of every sequence, lengths with them; rows of T tokens, `before` and `behind` of which belong to none."""

    def __init__(self, seed, lengths, counts, heads, kv_heads, dim, page_size, dtype=torch.bfloat16, order="heads", rotary=None,
                 ragged=True, before=0, behind=0, positions=None):
        self.gen = gen = torch.Generator().manual_seed(seed)
        self.lengths, self.counts, self.page, self.dtype = lengths, counts, page_size, dtype
        rotary = dim if rotary is None else rotary
        T = before + sum(counts) + behind if ragged else len(lengths)
        rows = torch.randn(T, heads + 2 * kv_heads, dim, generator=gen).bfloat16()
        self.q, self.k, self.v = rows.split([heads, kv_heads, kv_heads], 1)
        self.rows = rows
        self.starts = torch.tensor([before + sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32) if ragged else None
        n_pages = sum(-(-n // page_size) for n in lengths) + 2
        self.table = page_table(lengths, page_size, n_pages, gen)
        self.cos_sin = angles(max(1, max(lengths)) if positions is None else positions, rotary)
        shape = (n_pages, page_size, kv_heads, dim)
        fill = lambda: torch.randint(-100, 100, shape, generator=gen).to(dtype)
        self.cache = [fill(), fill()]
        self.scales = [torch.randn(n_pages, kv_heads, page_size, generator=gen) for _ in range(2)] if dtype == torch.int8 else [None, None]
        self.order = order

    def on_gpu(self):
        put = lambda x: x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.order == "heads" else x.cuda()
        ks, vs = (None if s is None else s.clone().cuda() for s in self.scales)
        return binding.KVCache(put(self.cache[0].clone()), put(self.cache[1].clone()), self.table.cuda(), ks, vs)

    def args(self):
        q, k, v = self.rows.cuda().split([self.q.shape[1], self.k.shape[1], self.k.shape[1]], 1)
        return q, k, v, self.cos_sin.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(), \
            None if self.starts is None else self.starts.cuda()

    def tokens(self):
        """(row, sequence, position) of every token that has a place."""
        for b, n in enumerate(self.lengths):
            if self.starts is None:
                if n:
                    yield b, b, n - 1
            else:
                for i in range(self.counts[b]):
                    if n:
                        yield int(self.starts[b]) + i, b, n - self.counts[b] + i

    def expected(self, interleaved=False):
        """q_out, the caches and their scales as they should be: values in fp64, how far a bf16 may be off, codes and scales exactly."""
        row, seq, pos = (torch.tensor(x, dtype=torch.long) for x in zip(*self.tokens()))
        page = self.table[seq, pos // self.page].long()
        at = pos % self.page
        R = self.cos_sin.shape[1]
        c, s = self.cos_sin[pos, None, :R // 2].double(), self.cos_sin[pos, None, R // 2:].double()
        a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))

        def turned(x):
            y, size = x.double(), x.double().abs()
            u, w = y[..., a].clone(), y[..., b].clone()
            y[..., a], y[..., b] = u * c - w * s, w * c + u * s
            size[..., a], size[..., b] = (u * c).abs() + (w * s).abs(), (w * c).abs() + (u * s).abs()
            return y, BF16_HALF_STEP * y.abs() + 4 * H * size + 1e-38     # three roundings to binary32, one to bf16
        out = {"q": (row, *turned(self.q[row]))}
        if self.dtype == torch.int8:
            k32 = rotated32(self.k[row].float().numpy(), self.cos_sin[pos].numpy(), interleaved)
            out["codes"] = [quantized(x) for x in (k32, self.v[row].float().numpy())]
        else:
            out["k"] = turned(self.k[row])
            out["v"] = self.v[row]
        return out, page, at


def check(batch, interleaved=False, q_out=None):
    cache, (q, k, v, cos_sin, lens, starts) = batch.on_gpu(), batch.args()
    given = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda") if q_out is None else q_out
    got = binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=given, interleaved=interleaved)
    binding.check_status()
    assert got is given
    want, page, at = batch.expected(interleaved)
    row, y, tol = want["q"]
    assert_within(got[row.cuda()], y, tol, "q")
    others = torch.ones(got.shape[0], dtype=torch.bool)
    others[row] = False
    assert (got[others.cuda()] == 7).all()
    for i, name in enumerate("kv"):
        before, after = batch.cache[i], (cache.k, cache.v)[i].cpu()
        keep = torch.ones(before.shape[:2], dtype=torch.bool)
        keep[page, at] = False
        assert torch.equal(after[keep], before[keep]), name + ": other places"
        if batch.dtype == torch.int8:
            codes, scales = want["codes"][i]
            after_scales = (cache.k_scales, cache.v_scales)[i].cpu().transpose(1, 2)
            assert np.array_equal(after[page, at].numpy(), codes), name
            assert np.array_equal(after_scales[page, at].numpy(), scales), name + " scales"
            assert torch.equal(after_scales[keep], batch.scales[i].transpose(1, 2)[keep])
        elif name == "k":
            assert_within(after[page, at], *want["k"], "k")
        else:
            assert torch.equal(after[page, at], want["v"])
    return got, cache


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (20, 4), (71, 1), (64, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_one_token_per_sequence(dtype, dim, heads, kv_heads, interleaved):
    check(Batch(dim + heads, [1, 17, 0, 16, 300], [1, 1, 0, 1, 1], heads, kv_heads, dim, 16, dtype, ragged=False), interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("page_size", [1, 3, 16, 100])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_prompts_and_pieces(dtype, page_size, order):
    """A whole prompt, the last piece of another, one token, none, and rows of no sequence before and behind."""
    check(Batch(page_size, [37, 90, 5, 12, 0], [37, 33, 1, 0, 0], 8, 2, 128, page_size, dtype, order, before=3, behind=5))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("rotary", [16, 32, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_partial_rotation(dtype, rotary, interleaved):
    check(Batch(rotary, [20, 33], [9, 33], 6, 3, 128, 16, dtype, rotary=rotary), interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("tokens", [1, 700, 2500])
def test_few_tokens_and_many(dtype, tokens):
    check(Batch(tokens, [tokens + 11, 3], [tokens, 2], 10, 5, 64, 32, dtype))


@pytest.mark.gpu
def test_many_sequences():
    counts = [(7 * i) % 4 for i in range(700)]
    check(Batch(3, [c + i % 5 if c else 0 for i, c in enumerate(counts)], counts, 4, 2, 64, 8))


@pytest.mark.gpu
def test_far_positions():
    """The last of 200000 positions: its angles are the table's, whatever their size."""
    check(Batch(4, [200000, 199984], [40, 1], 2, 1, 64, 512))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_heads_of_zeros_and_of_no_numbers(dtype):
    batch = Batch(5, [4, 9], [4, 9], 2, 2, 64, 16, dtype)
    batch.rows[2] = 0
    batch.rows[3, :, 5] *= 1e30
    check(batch)                                           # (zeros: a scale of 1 and codes of 0)
    if dtype == torch.int8:
        cache, args = batch.on_gpu(), list(batch.args())
        args[1] = args[1].clone()
        args[1][6, 1, 3], args[1][7, 0, 3] = math.nan, math.inf
        binding.kv_append(cache, *args[:4], args[4], args[5])
        page, at = places(batch.table, 1, [2, 3], 16)
        scales = cache.k_scales.cpu().transpose(1, 2)[page, at]
        assert not scales[0, 1].isfinite() and not scales[1, 0].isfinite()
        assert scales[0, 0].isfinite() and scales[1, 1].isfinite()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_in_place_new_and_without_queries(dtype):
    batch = Batch(6, [30, 8, 0], [30, 3, 0], 6, 2, 128, 16, dtype, behind=2)
    given, cache = check(batch)
    live = given != 7
    q, k, v, cos_sin, lens, starts = batch.args()
    fresh = binding.kv_append(batch.on_gpu(), q, k, v, cos_sin, lens, starts)
    assert torch.equal(fresh[live], given[live]) and (fresh[~live] == 0).all()
    again = batch.on_gpu()
    kept = q.clone()
    assert binding.kv_append(again, q, k, v, cos_sin, lens, starts, q_out=q) is q
    assert torch.equal(q[live], given[live]) and torch.equal(q[~live], kept[~live])
    alone = batch.on_gpu()
    assert binding.kv_append(alone, None, k, v, cos_sin, lens, starts) is None
    for c in (again, alone):
        assert torch.equal(c.k, cache.k) and torch.equal(c.v, cache.v)
    binding.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["page too high", "page below 0", "length too high", "length below 0", "too few angles", "length below the new tokens"])
def test_what_is_out_of_range_is_noted_and_left_out(what):
    batch = Batch(7, [40, 25, 60], [10, 25, 1], 4, 2, 64, 16)
    cache, (q, k, v, cos_sin, lens, starts) = batch.on_gpu(), batch.args()
    good = batch.on_gpu()
    binding.kv_append(good, q, k, v, cos_sin, lens, starts)
    binding.check_status()
    if what.startswith("page"):
        cache.page_table[1, 0] = cache.k.shape[0] if what.endswith("high") else -1
    elif what == "too few angles":
        cos_sin = cos_sin[:59].contiguous()
    else:
        lens[1] = {"h": cache.page_table.shape[1] * 16 + 1, "0": -25, "s": 24}[what[-1]]
    q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=q_out)
    with pytest.raises(binding.PeqaError) as err:
        binding.check_status()
    assert err.value.status == -10
    # the other sequences' tokens have their places, and what has none is nowhere
    for b in (0, 1, 2):
        if b == (2 if what == "too few angles" else 1):
            continue
        page, at = places(batch.table, b, range(batch.lengths[b] - batch.counts[b], batch.lengths[b]), 16)
        assert torch.equal(cache.k[page, at], good.k[page, at]) and torch.equal(cache.v[page, at], good.v[page, at])
    binding.check_status()


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    batch = Batch(8, [30, 8, 64], [1, 1, 1], 8, 2, 128, 16, ragged=False)
    q, k, v, cos_sin, lens, _ = batch.args()
    cache = batch.on_gpu()
    q_out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    append = lambda c, **kw: binding.kv_append(c, q, k, v, cos_sin, lens, **kw)
    append(cache, q_out=q_out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        append(cache, q_out=q_out)
    other = torch.cuda.Stream()
    for lengths in ([29, 0, 50], [2, 7, 0]):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        fresh = batch.on_gpu()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            want = append(fresh)
        torch.cuda.synchronize()
        for b, n in enumerate(lengths):
            if n:
                page, at = places(batch.table, b, [n - 1], 16)
                assert torch.equal(cache.k[page, at], fresh.k[page, at]) and torch.equal(q_out[b], want[b])
    binding.check_status()


@pytest.mark.gpu
def test_refusals():
    batch = Batch(9, [30, 8, 64], [1, 1, 1], 8, 2, 128, 16, ragged=False)
    cache, (q, k, v, cos_sin, lens, _) = batch.on_gpu(), batch.args()
    starts = torch.arange(4, dtype=torch.int32, device="cuda")
    append = binding.kv_append
    for args in ((q, k[:, :1], v, cos_sin, lens), (q, k, v[:2], cos_sin, lens), (q, k[:2], v[:2], cos_sin, lens), (q.float(), k, v, cos_sin, lens),
                 (q, k, v, cos_sin.double(), lens), (q, k, v, cos_sin[0], lens), (q, k, v, cos_sin, lens.long()), (q, k, v, cos_sin, lens[:2]),
                 (q, k, v, cos_sin, lens, starts[:3]), (q[:2], k, v, cos_sin, lens), (q, k, v, cos_sin.cpu(), lens)):
        with pytest.raises(ValueError):
            append(cache, *args)
    for q_out in (q[:, :4], torch.zeros_like(q, dtype=torch.float32)):
        with pytest.raises(ValueError):
            append(cache, q, k, v, cos_sin, lens, q_out=q_out)
    with pytest.raises(ValueError):
        append(cache, None, k, v, cos_sin, lens, q_out=torch.empty_like(q))
    for bad in (angles(64, 8), angles(64, 136)):
        with pytest.raises(binding.PeqaError) as err:
            append(cache, q, k, v, bad.cuda(), lens)
        assert err.value.status == -3
    with pytest.raises(binding.PeqaError) as err:
        append(cache, q, k, v, cos_sin, lens, q_out=torch.empty(8, 128, dtype=torch.bfloat16, device="cuda").expand(3, 8, 128))
    assert err.value.status == -3
    assert torch.equal(cache.k.cpu(), batch.cache[0]) and torch.equal(cache.v.cpu(), batch.cache[1])
    binding.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("what", ["in place", "page too high", "page below 0", "length too high", "length below 0", "length below the new tokens"])
def test_runs_of_many_tokens(dtype, what):
    """In place, and with one sequence that is out of range (a page: some of its tokens)."""
    batch = Batch(11, [2000, 300, 1500], [1900, 290, 1400], 4, 2, 128, 16, dtype, behind=3)
    cache, (q, k, v, cos_sin, lens, starts) = batch.on_gpu(), batch.args()
    good = batch.on_gpu()
    want = binding.kv_append(good, q, k, v, cos_sin, lens, starts)
    binding.check_status()
    if what == "in place":
        kept = q.clone()
        binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=q)
        assert torch.equal(q[:-3], want[:-3]) and torch.equal(q[-3:], kept[-3:])
    else:
        if what.startswith("page"):
            cache.page_table[1, 5] = cache.k.shape[0] if what.endswith("high") else -1
        else:
            lens[1] = {"h": cache.page_table.shape[1] * 16 + 1, "0": -25, "s": 289}[what[-1]]
        got = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=got)
        with pytest.raises(binding.PeqaError) as err:
            binding.check_status()
        assert err.value.status == -10
        for first, end in ((0, 1900), (2190, 3590)):
            assert torch.equal(got[first:end], want[first:end])
        if what.startswith("length") and what[-1] != "s":
            assert (got[1900:2190] == 7).all()
    for b in (0, 2) if what != "in place" else (0, 1, 2):
        page, at = places(batch.table, b, range(batch.lengths[b]), 16)
        assert torch.equal(cache.k[page, at], good.k[page, at]) and torch.equal(cache.v[page, at], good.v[page, at])
    binding.check_status()


@pytest.mark.gpu
def test_captured_pieces_follow_their_starts():
    """A captured call of a fixed number of rows, replayed with other pieces and lengths."""
    batch = Batch(12, [90, 80, 100], [20, 10, 10], 6, 2, 64, 16, behind=8)
    q, k, v, cos_sin, lens, starts = batch.args()
    cache, q_out = batch.on_gpu(), torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=q_out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=q_out)
    for lengths, bounds in (([33, 0, 48], [0, 33, 33, 48]), ([34, 80, 49], [5, 6, 40, 41]), ([90, 1, 100], [0, 20, 20, 20])):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        starts.copy_(torch.tensor(bounds, dtype=torch.int32))
        q_out.zero_()
        for x, y in zip((cache.k, cache.v), batch.cache):
            x.copy_(y)
        g.replay()
        fresh = batch.on_gpu()
        want = binding.kv_append(fresh, q, k, v, cos_sin, lens, starts)
        assert torch.equal(q_out, want) and torch.equal(cache.k, fresh.k) and torch.equal(cache.v, fresh.v)
    binding.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim,tokens", [(64, 2900), (128, 1500), (256, 800)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_many_heads_of_many_tokens(dtype, dim, tokens, interleaved):
    """Enough for 8-bit caches to take tokens in runs; a part of the channels turns."""
    check(Batch(dim, [tokens + 300, 9, 0, 40], [tokens, 1, 0, 40], 70, 13, dim, 16, dtype, rotary=dim - 16, before=2, behind=1), interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [31, 32, 33, 1023, 1025, 2100])
def test_one_token_of_many_sequences_and_pieces(seqs):
    """With and without starts, sequences of none among them; the search for a row's sequence ends at 32, 1024, ..."""
    counts = [(5 * i) % 3 for i in range(seqs)]
    check(Batch(seqs, [c + i % 7 if c else 0 for i, c in enumerate(counts)], counts, 2, 1, 64, 4, before=3, behind=2))
    check(Batch(seqs, [(3 * i) % 5 for i in range(seqs)], [1] * seqs, 2, 1, 64, 4, ragged=False))


@pytest.mark.gpu
@pytest.mark.parametrize("ragged", [False, True])
def test_many_sequences_of_an_8_bit_cache_in_runs(ragged):
    n = 1500
    counts = [1 if i % 9 else 0 for i in range(n)] if ragged else [1] * n
    check(Batch(13, [c + i % 4 if c else 0 for i, c in enumerate(counts)], counts, 80, 16, 128, 8, torch.int8, ragged=ragged))


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["in place", "page too high", "page below 0", "length too high", "length below 0", "length below the new tokens"])
def test_runs_of_an_8_bit_cache(what):
    """In place, and with one sequence that is out of range (a page: some of its tokens)."""
    batch = Batch(14, [900, 300, 900], [800, 290, 700], 64, 8, 128, 16, torch.int8, behind=3)
    cache, (q, k, v, cos_sin, lens, starts) = batch.on_gpu(), batch.args()
    good = batch.on_gpu()
    want = binding.kv_append(good, q, k, v, cos_sin, lens, starts)
    binding.check_status()
    if what == "in place":
        kept = q.clone()
        binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=q)
        assert torch.equal(q[:-3], want[:-3]) and torch.equal(q[-3:], kept[-3:])
    else:
        if what.startswith("page"):
            cache.page_table[1, 5] = cache.k.shape[0] if what.endswith("high") else -1
        else:
            lens[1] = {"h": cache.page_table.shape[1] * 16 + 1, "0": -25, "s": 289}[what[-1]]
        got = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        binding.kv_append(cache, q, k, v, cos_sin, lens, starts, q_out=got)
        with pytest.raises(binding.PeqaError) as err:
            binding.check_status()
        assert err.value.status == -10
        for first, end in ((0, 800), (1090, 1790)):
            assert torch.equal(got[first:end], want[first:end])
        if what.startswith("length") and what[-1] != "s":
            assert (got[800:1090] == 7).all()
    for b in (0, 2) if what != "in place" else (0, 1, 2):
        page, at = places(batch.table, b, range(batch.lengths[b]), 16)
        assert torch.equal(cache.k[page, at], good.k[page, at]) and torch.equal(cache.v[page, at], good.v[page, at])
    binding.check_status()
