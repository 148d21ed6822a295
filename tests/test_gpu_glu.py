"""The gated feed-forward block against its definition in 64 bits: forward, backward, single tokens, and a step of them together."""
import pytest
import torch

from glu_util import backward, block, forward
from loss_util import assert_within
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu

#: tokens, channels, columns: tiles cut everywhere, few and many tokens (both kernels), rows of H that begin at 16 bytes and at 32
SHAPES = [(1, 8, 128), (5, 24, 256), (16, 136, 384), (17, 40, 128), (77, 1000, 512), (200, 264, 1024), (513, 1048, 128), (300, 2048, 640),
          (1030, 520, 256), (2100, 1376, 512)]


def rows(T, K, seed):
    return torch.randn((T, K), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("T,F,K", SHAPES)
def test_forward(T, F, K, group, bits):
    w, W, _ = block(F, K, bits, group, seed=F + K)
    X = rows(T, K, T)
    act = "silu" if (T + bits) % 2 else "gelu_tanh"
    H, Y = binding.qglu_fwd(w, X, act)
    alone, none = binding.qglu_fwd(w, X, act, keep=False)
    assert none is None and torch.equal(H, alone)
    if w.G == 1:
        assert torch.equal(Y, binding.qlinear_fwd(w, X))
    binding.check_status()
    want, want_Y, tol, tol_Y = forward(X, W, act, w.G > 1)
    assert_within(Y, want_Y, tol_Y, "Y")
    assert_within(H, want, tol, "H")


#: row tiles (of 128) that a few clusters are left with behind whole waves of 148
WIDE = [(33, 10240, 1024), (77, 9480, 1024), (200, 10240, 512)]


@pytest.mark.parametrize("bits,group", [(4, 0), (4, 128), (3, 64)])
@pytest.mark.parametrize("T,F,K", WIDE)
def test_forward_of_a_wide_block(T, F, K, bits, group):
    w, W, _ = block(F, K, bits, group, seed=F)
    X = rows(T, K, T)
    H, Y = binding.qglu_fwd(w, X)
    alone, _ = binding.qglu_fwd(w, X, keep=False)
    assert torch.equal(H, alone)
    binding.check_status()
    want, want_Y, tol, tol_Y = forward(X, W, "silu", w.G > 1)
    assert_within(Y, want_Y, tol_Y, "Y")
    assert_within(H, want, tol, "H")


@pytest.mark.parametrize("group", [0, 128])
def test_wide_blocks_one_behind_another(group):
    """Every call reads what the one before has written, eagerly and captured, and no result is left to timing."""
    T, F, K = 33, 10240, 1024
    up, _, _ = block(F, K, 4, group, seed=1)
    down, _, _ = block(K // 2, F, 4, group, seed=2)
    X = rows(T, K, 3)
    H = torch.empty((T, F), dtype=torch.bfloat16, device="cuda")
    Z = torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
    space = binding.alloc_workspace(binding.OP_GLU_FWD, T, up)

    def chain(pause):
        Z.copy_(X)
        for _ in range(6):
            binding.qglu_fwd(up, Z, keep=False, H=H, workspace=space)
            pause()
            binding.qlinear_fwd(down, H, Z)
            pause()

    chain(torch.cuda.synchronize)
    want = Z.clone()
    assert want.isfinite().all()
    chain(lambda: None)
    assert torch.equal(Z, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(lambda: None)
    for _ in range(5):
        Z.zero_()
        graph.replay()
        assert torch.equal(Z, want)
    binding.check_status()


@pytest.mark.parametrize("T,F,K", [(9, 40, 64), (100, 88, 192), (700, 72, 320)])
def test_forward_of_odd_multiples_of_64_columns(T, F, K):
    w, W, _ = block(F, K, 4, 64, seed=3)
    X = rows(T, K, 4)
    H, Y = binding.qglu_fwd(w, X)
    want, want_Y, tol, tol_Y = forward(X, W, "silu", w.G > 1)
    assert_within(Y, want_Y, tol_Y, "Y")
    assert_within(H, want, tol, "H")


@pytest.mark.parametrize("T", [30, 600])
def test_forward_of_scales_and_tokens_of_any_size(T):
    """Rows whose scales are far apart, or all 0; tokens from 2^-100 to 2^100, of zeros, with channels far below the largest."""
    F, K = 40, 512
    w, _, codes = block(F, K, 4, 64, seed=50)
    w.scales *= 2.0 ** (torch.arange(2 * F, device="cuda") % 40 - 20)[:, None]
    w.scales[:, 1::2] *= 2.0 ** -9
    w.scales[16:24] = 0
    from glu_util import weights
    W = weights(codes, w.zeros, w.scales)
    X = (rows(T, K, 51) * 2.0 ** (10 * (torch.arange(T, device="cuda") % 5 - 2))[:, None]).bfloat16()
    X[3] *= 2.0 ** -80
    X[4] = 0
    X[5, ::2] *= 2.0 ** -20
    H, Y = binding.qglu_fwd(w, X)
    want, want_Y, tol, tol_Y = forward(X, W, "silu", True)
    assert_within(Y, want_Y, tol_Y + 2.0 ** -126, "Y")
    near = want_Y.abs().amax(1) < 2.0 ** 60                    # products within binary32
    assert_within(H[near], want[near], tol[near] + 2.0 ** -126, "H")
    X[7, 9], X[8, 9] = float("inf"), float("nan")
    Y2 = binding.qglu_fwd(w, X)[1]
    assert not Y2[7:9, w.scales.amax(1) > 0].isfinite().all() and Y2[8].isnan().all()
    keep = [t for t in range(T) if t not in (7, 8)]
    assert torch.equal(Y2[keep], Y[keep])


@pytest.mark.parametrize("T,F", [(40, 520), (1500, 520), (40, 264), (1500, 264)])
def test_forward_writes_what_it_is_given_and_no_more(T, F):
    """Outputs inside larger buffers, H at an odd multiple of 16 bytes."""
    w, _, _ = block(F, 256, 4, 0, seed=5)
    X = rows(T, 256, 6)
    want, want_Y = binding.qglu_fwd(w, X)
    for lead in (8, 16):
        buf = torch.full((lead + T * F + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        buf_Y = torch.full((lead + 2 * T * F + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        H, Y = buf[lead:lead + T * F].view(T, F), buf_Y[lead:lead + 2 * T * F].view(T, 2 * F)
        binding.qglu_fwd(w, X, Y=Y, H=H)
        assert torch.equal(H, want) and torch.equal(Y, want_Y)
        for b, n in ((buf, T * F), (buf_Y, 2 * T * F)):
            assert (b[:lead] == 7).all() and (b[lead + n:] == 7).all()


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("T,F", [(1, 8), (3, 1000), (1001, 264), (64, 4096)])
def test_backward_of_the_activation(T, F, act):
    gen = torch.Generator(device="cuda").manual_seed(T + F)
    Y = (2 * torch.randn((T, 2 * F), generator=gen, device="cuda")).bfloat16()
    dH = torch.randn((T, F), generator=gen, device="cuda").bfloat16()
    # where exponentials over- and underflow, and where nothing happens
    odd = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 80.0, -80.0, 1e4, -1e4, 3e19, -3e19, 1e-3, -1.28, -5.5, 5.5, -0.75, 0.75], device="cuda")
    for i, v in enumerate(odd.tolist()):
        Y[i % T, (16 * i + i % 8) % (2 * F)] = v
    dY = binding.glu_bwd(Y, dH, act)
    want, tol = backward(Y, dH, act)
    assert not dY.isnan().any()
    fine = want.isfinite()                                    # autograd's own inf * 0 far out
    assert_within(torch.where(fine, dY, 0), torch.where(fine, want, 0), torch.where(fine, tol, 0), "dY")
    over = Y.clone()
    assert binding.glu_bwd(over, dH, act, dY=over).data_ptr() == over.data_ptr()
    assert torch.equal(over, dY)


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("group", [0, 64, 128, 256, 512])
@pytest.mark.parametrize("F,K", [(8, 512), (24, 1024), (1000, 512), (5504, 2048)])
def test_decode(F, K, group, bits):
    w, W, _ = block(F, K, bits, group, seed=F + group)
    prepared = binding.decode_prepare(w)
    torch.cuda.synchronize()
    for M in (1, 2, 3, 7, 8, 9, 13, 16):
        X = rows(M, K, M)
        act = "gelu_tanh" if M % 2 else "silu"
        H = binding.qglu_decode_prepared(w, prepared, X, act)
        want, _, tol, _ = forward(X, W, act, False)
        assert_within(H, want, tol, f"H of {M}")
    binding.check_status()


@pytest.mark.parametrize("bits,group", [(3, 0), (3, 128), (4, 64), (4, 256)])
@pytest.mark.parametrize("F,K", [(40, 512), (3000, 1024)])
def test_decode_of_several_tasks(F, K, bits, group):
    w, _, codes = block(F, K, bits, group, seed=8)
    from glu_util import weights
    table = torch.stack([w.scales, 2 * w.scales, w.scales.flip(0)]).contiguous()
    prepared = binding.decode_prepare(w)
    torch.cuda.synchronize()
    for M in (1, 2, 5, 8, 11, 16):
        X = rows(M, K, M)
        ids = torch.arange(M, device="cuda", dtype=torch.int32) * 2 % 3
        H = binding.qglu_decode_prepared(w, prepared, X, scale_table=table, task_ids=ids)
        for t in range(3):
            mine = ids == t
            want, _, tol, _ = forward(X[mine], weights(codes, w.zeros, table[t]), "silu", False)
            assert_within(H[mine], want, tol, f"H of task {t}")


def test_rows_of_two_projections():
    gen = torch.Generator(device="cuda").manual_seed(1)
    Wg, Wu = (torch.randn((48, 256), generator=gen, device="cuda") for _ in range(2))
    gate, up = binding.quantize_rtn(Wg, 4, 64), binding.quantize_rtn(Wu, 4, 64)
    both = binding.glu_interleave(gate, up)
    whole = binding.quantize_rtn(binding.glu_rows(Wg, Wu), 4, 64)
    for a, b in ((both.qweight, whole.qweight), (both.zeros, whole.zeros), (both.scales, whole.scales)):
        assert torch.equal(a, b)
    assert all(torch.equal(a, b) for a, b in zip(binding.glu_split(both.scales), (gate.scales, up.scales)))
    X = rows(33, 256, 2)
    H, Y = binding.qglu_fwd(both, X)
    Yg, Yu = binding.glu_split(Y.T.contiguous())
    # the same sums in another order: a step of bf16 of Y, at most
    for got, one in ((Yg.T, gate), (Yu.T, up)):
        assert (got.double() - binding.qlinear_fwd(one, X).double()).abs().max() <= 2.0 ** -7 * Y.abs().max()


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("bits,group", [(4, 0), (3, 128)])
def test_a_training_step_to_the_loss(bits, group):
    """Block, down projection, residual, loss and back, the scales stepped; against autograd in 64 bits.  A dozen bf16 roundings, each
    off by 2^-9 in the mean, add up to less than 12 * 2^-9 of the whole; folded scales take two more a product."""
    T, K, F, V = 300, 256, 512, 3000
    w, W, codes = block(F, K, bits, group, seed=20)
    down_codes = torch.randint(2 ** bits, (K, F), device="cuda", generator=torch.Generator(device="cuda").manual_seed(21)).to(torch.uint8)
    G = 1 if group == 0 else F // group
    down = binding.QWeight(bits, K, F, group, binding.pack(down_codes, bits), torch.full((K, G), 2 ** (bits - 1), dtype=torch.uint8, device="cuda"),
                           torch.full((K, G), F ** -0.5 * 3.5 / 2 ** bits, device="cuda"))
    X = rows(T, K, 22)
    head = (rows(V, K, 23).float() * K ** -0.5).bfloat16()
    labels = torch.randint(V, (T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(24)).int()
    labels[::3] = -1
    weight = torch.full((T,), 1.0 / int((labels >= 0).sum()), device="cuda")

    H, Y = binding.qglu_fwd(w, X)
    Z = binding.qlinear_fwd(down, H) + X
    loss, dZ = binding.head_loss(Z, head, labels, weight)
    dH, dS_down = binding.qlinear_bwd(down, H, dZ)
    dY = binding.glu_bwd(Y, dH, dY=Y)
    dX, dS = binding.qlinear_bwd(w, X, dY)
    dX = dX + dZ
    binding.check_status()

    from glu_util import act, halves, weights
    s, s_down = w.scales.double().requires_grad_(), down.scales.double().requires_grad_()
    x = X.double().requires_grad_()

    def linear(x, codes, zeros, s):
        n, g = zeros.shape
        q = codes.double().view(n, g, -1) - zeros.double()[:, :, None]
        return x @ (q * s[:, :, None]).view(n, -1).T

    gate, up = halves(linear(x, codes, w.zeros, s))
    z = linear(act(gate, "silu") * up, down_codes, down.zeros, s_down) + x
    live = labels >= 0
    each = torch.nn.functional.cross_entropy((z @ head.double().T)[live], labels[live].long(), reduction="none")
    (each * weight[live].double()).sum().backward()
    assert _rel(loss[live], each.detach()) < 12 * 2.0 ** -9
    for got, want in ((dX, x.grad), (dS, s.grad), (dS_down, s_down.grad)):
        assert _rel(got, want) < 16 * 2.0 ** -9
    m, v = torch.zeros_like(w.scales), torch.zeros_like(w.scales)
    before = w.scales.clone()
    binding.qlinear_bwd_ds_adamw(w, X, dY, m, v, lr=1e-5)
    assert not torch.equal(before, w.scales) and w.scales.isfinite().all()


def test_what_is_refused():
    w, _, _ = block(64, 256, 4, 64, seed=40)
    X = rows(20, 256, 41)
    ws = binding.alloc_workspace(binding.OP_GLU_FWD, 20, w)
    for bad, status in ((ws[:-256], -5), (torch.cat([ws, ws])[16:], -4)):
        with pytest.raises(binding.PeqaError) as e:
            binding.qglu_fwd(w, X, workspace=bad)
        assert e.value.status == status
    X, H = rows(20, 256, 41), torch.zeros((20, 64), dtype=torch.bfloat16, device="cuda")
    Y = torch.zeros((20, 128), dtype=torch.bfloat16, device="cuda")
    prepared = binding.decode_prepare(w)
    torch.cuda.synchronize()
    few = X[:4].contiguous()
    for call in (lambda: binding.qglu_fwd(w, X[:, :128].contiguous()), lambda: binding.qglu_fwd(w, X.float()), lambda: binding.qglu_fwd(w, X.cpu()),
                 lambda: binding.qglu_fwd(w, X, "relu"), lambda: binding.qglu_fwd(w, X, 0), lambda: binding.qglu_fwd(w, X, H=Y),
                 lambda: binding.qglu_fwd(w, X, Y=H), lambda: binding.glu_bwd(Y, H[:19]), lambda: binding.glu_bwd(Y, Y),
                 lambda: binding.glu_bwd(Y, H, dY=H), lambda: binding.glu_bwd(Y, H, "gelu"), lambda: binding.glu_bwd(Y[:, :64], H),
                 lambda: binding.qglu_decode_prepared(w, prepared[:-1], few), lambda: binding.qglu_decode_prepared(w, prepared, few, scale_table=w.scales[None]),
                 lambda: binding.qglu_decode_prepared(w, prepared, few, scale_table=w.scales[None, :-1].contiguous(), task_ids=torch.zeros(4, dtype=torch.int32, device="cuda")),
                 lambda: binding.qglu_decode_prepared(w, prepared, few, scale_table=w.scales[None], task_ids=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(binding.PeqaError) as e:
        binding.qglu_decode_prepared(w, prepared, X)
    assert e.value.status == -3                               # more than 16 tokens
    binding.check_status()


def test_captured_decode_beside_another_stream():
    w, _, _ = block(1024, 1024, 3, 64, seed=30)
    prepared = binding.decode_prepare(w)
    torch.cuda.synchronize()
    X, other = rows(4, 1024, 31), rows(300, 1024, 32)
    want, want_other = binding.qglu_decode_prepared(w, prepared, X).clone(), binding.qglu_fwd(w, other)[0].clone()
    H = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.qglu_decode_prepared(w, prepared, X, H=H)
    side = torch.cuda.Stream()
    for _ in range(5):
        H.zero_()
        graph.replay()
        with torch.cuda.stream(side):
            got = binding.qglu_fwd(w, other)[0]
        torch.cuda.synchronize()
        assert torch.equal(H, want) and torch.equal(got, want_other)
