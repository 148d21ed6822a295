"""What the gated block's entry points refuse before they touch a device."""
import ctypes

import pytest
import torch

from paper_2305_14152_b200 import binding, build

NULL, BITS, SHAPE, ALIGN, LARGE = -1, -2, -3, -4, -9


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(4096)
    yield (ctypes.addressof(buf) + 255) & ~255
    del buf


def weight(p, bits=4, N=64, K=256, group=0, **more):
    return ctypes.byref(binding._QWeight(bits, N, K, group, more.get("q", p), more.get("z", p), more.get("s", p)))


def test_forward(L, p):
    call = lambda w, act=0, X=p, T=4, Y=p, H=p: L.peqa_qglu_fwd(w, act, X, T, Y, H, p, 1 << 40, 0)
    w = weight(p)
    assert call(w, X=0) == NULL and call(w, H=0) == NULL and call(None) == NULL and call(weight(p, z=0)) == NULL
    assert call(w, X=p + 8) == ALIGN and call(w, H=p + 8) == ALIGN and call(w, Y=p + 8) == ALIGN
    assert call(weight(p, bits=2)) == BITS
    for bad in (weight(p, N=8), weight(p, N=72), weight(p, K=96), weight(p, bits=3, K=192), weight(p, group=48)):
        assert call(bad) == SHAPE
    assert call(w, T=0) == SHAPE and call(w, act=2) == SHAPE and call(w, act=-1) == SHAPE


def test_backward(L, p):
    call = lambda act=0, Y=p, dH=p, T=4, F=64, dY=p: L.peqa_glu_bwd(act, Y, dH, T, F, dY, 0)
    for name in ("Y", "dH", "dY"):
        assert call(**{name: 0}) == NULL and call(**{name: p + 8}) == ALIGN
    for bad in ({"T": 0}, {"F": 0}, {"F": 12}, {"F": -8}, {"act": 2}):
        assert call(**bad) == SHAPE
    assert call(T=2 ** 31 - 1, F=2 ** 20) == LARGE


def test_decode(L, p):
    call = lambda w, act=0, prepared=p, X=p, M=4, H=p, table=0, n=0, ids=0: L.peqa_qglu_decode_prepared(w, act, prepared, X, M, H, table, n, ids, 0)
    w = weight(p)
    assert call(w, prepared=0) == NULL and call(w, X=0) == NULL and call(w, H=0) == NULL and call(weight(p, s=0)) == NULL
    assert call(w, table=0, n=2, ids=p) == NULL and call(w, table=p, n=0, ids=p) == SHAPE
    assert call(w, M=0) == SHAPE and call(w, M=17) == SHAPE and call(w, act=7) == SHAPE
    assert call(weight(p, N=72)) == SHAPE and call(weight(p, K=192)) == SHAPE and call(weight(p, group=32)) == SHAPE
    assert call(w, H=p + 8) == ALIGN and call(w, prepared=p + 4) == ALIGN


def test_binding():
    y, h = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(4, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous CUDA tensor"):
        binding.glu_bwd(y, h)
    with pytest.raises(ValueError):
        binding.glu_rows(torch.zeros(12, 3), torch.zeros(12, 3))
    with pytest.raises(ValueError):
        binding.glu_rows(torch.zeros(16, 3), torch.zeros(8, 3))
    with pytest.raises(ValueError):
        binding.glu_split(torch.zeros(24, 2))
    a, b = torch.arange(48).view(24, 2), -torch.arange(48).view(24, 2)
    both = binding.glu_rows(a, b)
    assert torch.equal(both[:8], a[:8]) and torch.equal(both[8:16], b[:8]) and torch.equal(both[40:], b[16:])
    assert all(torch.equal(x, y) for x, y in zip(binding.glu_split(both), (a, b)))
    q = lambda bits, K: binding.QWeight(bits, 24, K, 0, torch.zeros(24, K * bits // 32, dtype=torch.int32), torch.zeros(24, 1, dtype=torch.uint8),
                                        torch.zeros(24, 1))
    assert binding.glu_interleave(q(4, 128), q(4, 128)).N == 48
    with pytest.raises(ValueError):
        binding.glu_interleave(q(4, 128), q(3, 128))
