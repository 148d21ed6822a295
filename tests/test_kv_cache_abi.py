"""Host-side checks of the paged cache's entry points: what is refused is refused before anything reaches a GPU."""
import ctypes

import pytest
import torch

from paper_2305_14152_b200 import binding, build


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


@pytest.fixture
def p():
    buf = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(buf) + 255) & ~255


def _cache(p, **change):
    c = binding._KVCache(type=0, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, n_seqs=3, max_pages=5, page_stride=16 * 2 * 64,
                         token_stride=64, head_stride=16 * 64, k=p, v=p, k_scales=0, v_scales=0, page_table=p)
    for name, value in change.items():
        setattr(c, name, value)
    return ctypes.byref(c)


BAD = [({"k": 0}, -1), ({"v": 0}, -1), ({"page_table": 0}, -1), ({"type": 2}, -2), ({"type": 1}, -1), ({"n_pages": 0}, -3),
       ({"page_size": 0}, -3), ({"n_kv_heads": 0}, -3), ({"head_dim": 96}, -3), ({"n_seqs": 0}, -3), ({"max_pages": -1}, -3),
       ({"token_stride": 0}, -3), ({"head_stride": -1024}, -3), ({"token_stride": 68}, -4), ({"type": 1, "token_stride": 72}, -1),
       ({"head_stride": 512}, -3),                          # heads within one another
       ({"page_stride": 64}, -3), ({"page_stride": 1 << 35}, -9), ({"page_stride": 1 << 40}, -9),
       ({"max_pages": 1 << 28}, -9), ({"n_pages": 1 << 30, "page_stride": 16 * 2 * 64}, -9)]


@pytest.mark.parametrize("change,status", BAD)
def test_descriptors(L, p, change, status):
    rows = binding._Rows(p, 8 * 64, 64)
    r = ctypes.byref(rows)
    assert L.peqa_attn_decode(_cache(p, **change), r, 8, p, 1.0, 0, p, 0, p, 1 << 16, 0) == status
    assert L.peqa_kv_append(_cache(p, **change), r, 8, r, r, 3, p, 9, 64, 0, p, 0, r, 0) == status


NO_DEVICE = (-6, -7)                                        # past the checks of the arguments the next refusal is the missing device


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that only a missing device refuses")
def test_what_is_taken(L, p):
    rows = lambda *a: ctypes.byref(binding._Rows(*a))
    good, kv = rows(p, 512, 64), rows(p, 128, 64)
    attend = lambda cache: L.peqa_attn_decode(cache, good, 8, p, 1.0, 0, p, 0, p, 1 << 16, 0)
    for page, token, head in ((2048, 64, 1024), (2048, 128, 64), (64, 512, 256), (64, 256, 4096)):
        assert attend(_cache(p, page_stride=page, token_stride=token, head_stride=head)) in NO_DEVICE     # strides in any order
    assert attend(_cache(p, n_pages=1, n_kv_heads=1, page_stride=-3, head_stride=0)) in NO_DEVICE         # a stride of one thing says nothing
    append = lambda q=good, tokens=3, starts=0: L.peqa_kv_append(_cache(p), q, 8, kv, kv, tokens, p, 9, 64, 0, p, starts, good, 0)
    assert append() in NO_DEVICE and append(tokens=4, starts=p) in NO_DEVICE
    assert append(q=rows(p, 0, 64)) in NO_DEVICE                                                         # q may repeat a row


def test_attend(L, p):
    rows = lambda *a: ctypes.byref(binding._Rows(*a))
    good = rows(p, 512, 64)
    call = lambda q=good, heads=8, lens=p, window=0, out=p, lse=0, cache=_cache(p): \
        L.peqa_attn_decode(cache, q, heads, lens, 1.0, window, out, lse, p, 1 << 16, 0)
    assert L.peqa_attn_decode(None, good, 8, p, 1.0, 0, p, 0, p, 1 << 16, 0) == -1
    assert call(q=None) == -1 and call(lens=0) == -1 and call(out=0) == -1 and call(q=rows(0, 512, 64)) == -1
    assert call(heads=7) == -3 and call(heads=0) == -3 and call(window=-1) == -3
    assert call(q=rows(p + 8, 512, 64)) == -4 and call(q=rows(p, 508, 64)) == -4 and call(out=p + 2) == -4
    assert call(lens=p + 2) == -4 and call(lse=p + 1) == -4
    assert call(q=rows(p, -512, 64)) == -3
    # 31 bits for the tiles of all rows
    assert call(cache=_cache(p, n_seqs=1 << 20, max_pages=1 << 16)) == -9


def test_append(L, p):
    rows = lambda *a: ctypes.byref(binding._Rows(*a))
    good, kv = rows(p, 512, 64), rows(p, 128, 64)

    def call(cache=_cache(p), q=good, heads=8, k=kv, v=kv, tokens=3, angles=p, positions=9, rotary=64, lens=p, starts=0, q_out=good):
        return L.peqa_kv_append(cache, q, heads, k, v, tokens, angles, positions, rotary, 0, lens, starts, q_out, 0)

    assert call(k=None) == -1 and call(v=None) == -1 and call(angles=0) == -1 and call(lens=0) == -1
    assert call(q=None) == -1 and call(q_out=None) == -1
    assert call(tokens=4) == -3 and call(tokens=0) == -3                              # one per sequence, or starts
    for rotary in (0, 8, 24, 80, -16):
        assert call(rotary=rotary) == -3
    assert call(positions=0) == -3 and call(heads=0) == -3
    assert call(angles=p + 4) == -4 and call(k=rows(p, 132, 64)) == -4 and call(starts=p + 2) == -4
    assert call(q_out=rows(p, 512, 32)) == -3 and call(q_out=rows(p, 64, 64)) == -3   # rows of q_out in one another's place


def test_workspace(L, p):
    n = lambda heads, **c: L.peqa_attn_workspace_bytes(_cache(p, **c), heads)
    assert n(8) > 0 and n(8) % 16 == 0
    assert n(7) == 0 and n(0) == 0 and n(8, head_dim=96) == 0 and n(8, n_kv_heads=0) == 0
    assert L.peqa_attn_workspace_bytes(None, 8) == 0
    assert n(32, n_kv_heads=2, head_dim=128) > n(16, n_kv_heads=2, head_dim=128)      # 16 query heads a row
    # it does not grow with what the lengths may be
    assert n(8, n_seqs=1000, max_pages=100000) == n(8)


def test_refusals_of_the_binding_need_no_gpu():
    table = torch.zeros((1, 1), dtype=torch.int32)
    cache = binding.alloc_kv_cache(1, 16, 2, 64, table)
    assert cache.k.shape == (1, 16, 2, 64) and cache.k.stride(3) == 1 and cache.k_scales is None
    assert binding.alloc_kv_cache(2, 16, 3, 64, table, torch.int8).k_scales.shape == (2, 3, 16)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    lens = torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="cache.k: expected a tensor on the current CUDA device"):
        binding.attn_decode(cache, q, lens)
    with pytest.raises(ValueError, match="cache.k: expected a tensor on the current CUDA device"):
        binding.kv_append(cache, q, q[:, :2], q[:, :2], torch.zeros(9, 64), lens)
    with pytest.raises(AttributeError):
        binding.attn_decode(None, q, lens)


def test_heads_of_an_append_are_bounded(L, p):
    rows = lambda *a: ctypes.byref(binding._Rows(*a))
    call = lambda heads, kv: L.peqa_kv_append(_cache(p, n_kv_heads=kv, head_stride=64, token_stride=kv * 64, page_stride=kv * 64 * 16),
                                              rows(p, heads * 64, 64), heads, rows(p, kv * 64, 64), rows(p, kv * 64, 64), 3, p, 9, 64, 0, p, 0,
                                              rows(p, heads * 64, 64), 0)
    assert call((1 << 18) - 3, 2) == -9 and call(1, 1 << 17) == -9
