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


# ---- q_out beside q, k and v

def _append(q, k, v, q_out):
    """What becomes of the call without a GPU: None where nothing but the device is missing, else the refusal's text."""
    cache = _cache(kv_heads=k.shape[1], dim=k.shape[2], dtype=torch.bfloat16)
    with pytest.raises(ValueError) as err:
        binding.kv_append(cache, q, k, v, torch.zeros((9, 64)), torch.ones(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), q_out=q_out)
    return None if "on the current CUDA device" in str(err.value) else str(err.value)


OVER_Q, OVER_KV = "q_out: expected q itself or memory apart from q", "q_out: expected memory apart from k and v"


def test_outputs_over_what_is_read():
    T, H, KV, D = 5, 4, 2, 64
    rows = torch.zeros((T, H + 2 * KV, D), dtype=torch.bfloat16)
    q, k, v = rows.split([H, KV, KV], 1)
    assert _append(q, k, v, q) is None                                       # in place, k and v behind q in the rows of one matrix
    assert _append(q, k, v, torch.zeros_like(q)) is None
    assert _append(q, k, v, rows[:, 1:1 + H]) == OVER_Q                      # a head further
    assert _append(q, k, v, rows[:, KV:KV + H]) == OVER_Q
    assert _append(q, k, v, rows[:, 2 * KV:]) == OVER_KV
    assert _append(q, k, v, rows[:, H - 1:2 * H - 1]) == OVER_Q
    other = torch.zeros_like(rows)
    for x, y, z, out in ((other[:, :H], k, v, rows[:, 1:1 + H]), (other[:, :H], v, k, rows[:, 3:3 + H])):
        assert _append(x, y, z, out) == OVER_KV
    assert _append(other[:, :H], k, v, q) is None
    pool = torch.zeros((T + 2, H, D), dtype=torch.bfloat16)
    apart = torch.zeros((T, KV, D), dtype=torch.bfloat16)
    assert _append(pool[:T], apart, apart, pool[1:T + 1]) == OVER_Q          # a row further
    assert _append(pool[:T], apart, apart, pool[:T].transpose(0, 1).contiguous().transpose(0, 1)) is None
    assert _append(pool[:1], apart[:1], apart[:1], pool[1:2]) is None
    # q, k and v of a head side by side, and the heads outermost
    heads = torch.zeros((T, H, 3, D), dtype=torch.bfloat16)
    assert _append(heads[:, :, 0], heads[:, :, 1], heads[:, :, 2], heads[:, :, 0]) is None
    assert _append(heads[:, :, 0], heads[:, :, 1], heads[:, :, 1], heads[:, :, 2]) is None
    assert _append(heads[:, :, 0], heads[:, :, 1], heads[:, :, 2], heads[:, :, 1]) == OVER_KV
    outer = torch.zeros((H + 2 * KV, T, D), dtype=torch.bfloat16).transpose(0, 1)
    q, k, v = outer.split([H, KV, KV], 1)
    assert _append(q, k, v, q) is None and _append(q, k, v, outer[:, 1:1 + H]) == OVER_Q
    assert _append(q, q[:, :1].expand(T, KV, D), v, torch.zeros_like(q)) is None
    assert _append(q, k, v, q[:1].expand(T, H, D)) == OVER_Q


@pytest.mark.parametrize("same_rows", [True, False])
def test_overlaps_are_found_by_their_elements(same_rows):
    """Views of one buffer at random, against the lists of their elements.  Rows in one stride: refused where an element is in common and there
    alone.  Else nothing in common is taken that way, and what is refused lies within one extent."""
    gen = torch.Generator().manual_seed(21 + same_rows)
    ints = lambda hi: int(torch.randint(0, hi, (1,), generator=gen))
    pool = torch.zeros(40000, dtype=torch.bfloat16)
    places = torch.arange(pool.numel())
    found = {True: 0, False: 0}
    for _ in range(1500):
        T, D = 1 + ints(4), 64
        stride = 8 * (1 + ints(120))

        def view(heads):
            row = stride if same_rows else 8 * (1 + ints(120))
            size, strides, at = (T, heads, D), (row, 8 * (1 + ints(60)), 1), 8 * ints(200)
            return pool.as_strided(size, strides, at), set(places.as_strided(size, strides, at).flatten().tolist())

        (q, _), (k, _) = ((torch.zeros((T, n, D), dtype=torch.bfloat16), None) for n in (3, 2))
        out, its = view(3)
        read, others = view(3 if ints(2) else 2)
        got = _append(read, k, k, out) if read.shape[1] == 3 else _append(q, read, read, out)
        common = bool(its & others)
        within = max(its) >= min(others) and max(others) >= min(its)
        if read.data_ptr() == out.data_ptr() and read.stride() == out.stride() and read.shape == out.shape:
            continue
        refused = got is not None
        assert got in (None, OVER_Q if read.shape[1] == 3 else OVER_KV)
        assert refused == common if same_rows or T == 1 else (refused or not common) and (within or not refused), (out.stride(), read.stride())
        found[refused] += 1
    assert min(found.values()) > 100, found


@pytest.mark.gpu
def test_queries_in_place_beside_keys_and_values():
    """The rows of one projection: q is turned where it lies, k and v are what they were; an output over them is refused and nothing is written."""
    T, H, KV, D = 3, 4, 2, 64
    gen = torch.Generator().manual_seed(22)
    rows = torch.randn((T, H + 2 * KV, D), generator=gen).bfloat16().cuda()
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    cos_sin = torch.randn((32, D), generator=gen).cuda()
    lens = torch.tensor([5, 17, 32], dtype=torch.int32, device="cuda")
    q, k, v = rows.split([H, KV, KV], 1)
    kept = rows.clone()
    for bad in (rows[:, 1:1 + H], rows[:, 2 * KV:]):
        with pytest.raises(ValueError, match="q_out: expected"):
            binding.kv_append(binding.alloc_kv_cache(6, 16, KV, D, table), q, k, v, cos_sin, lens, q_out=bad)
    assert torch.equal(rows, kept)
    a, b = (binding.alloc_kv_cache(6, 16, KV, D, table) for _ in range(2))
    want = binding.kv_append(a, q, k, v, cos_sin, lens)
    assert binding.kv_append(b, q, k, v, cos_sin, lens, q_out=q) is q
    assert torch.equal(q, want) and torch.equal(rows[:, H:], kept[:, H:])
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    binding.check_status()
