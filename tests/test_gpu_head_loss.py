"""Loss of the vocabulary projection and its gradient against the definition in 64 bits."""
import pytest
import torch

from loss_util import assert_within, inputs, reference
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu

#: tokens, vocabulary, features: one of each, below, at and beyond the tiles of 256 and stages of 64, several pieces of the vocabulary, several
#: chunks of tokens
SHAPES = [(1, 1, 8), (1, 2, 64), (1, 1000, 64), (3, 257, 72), (17, 5000, 200), (150, 32000, 512), (255, 256, 256), (256, 513, 128),
          (257, 1025, 1000), (513, 2050, 136), (700, 50257, 96), (2048, 999, 2048), (8200, 9000, 64),
          (300, 1, 8), (300, 3, 40), (5, 270001, 64), (33, 333, 2056), (64, 32000, 128), (129, 8200, 640), (240, 4097, 328)]


def check(X, W, labels, weight, grad=True, **more):
    loss, dX = binding.head_loss(X, W, labels, weight, need_grad=grad, **more)
    binding.check_status()
    want, want_dX, tol, tol_dX = reference(X if more.get("dX") is not X else more["kept"], W, labels, weight)
    assert loss.dtype == torch.float32 and not loss.isnan().any()
    assert_within(loss, want, tol, "loss")
    if grad:
        assert dX.dtype == torch.bfloat16
        assert_within(dX, want_dX, tol_dX, "dX")
    else:
        assert dX is None


@pytest.mark.parametrize("T,V,K", SHAPES)
@pytest.mark.parametrize("grad", [True, False])
def test_against_the_definition(T, V, K, grad):
    check(*inputs(T, V, K, seed=T + V + K), grad=grad)


@pytest.mark.parametrize("ignored", [0.01, 0.6, 0.999, 1.1])
@pytest.mark.parametrize("T", [1, 31, 777])
def test_tokens_that_count_nothing(T, ignored):
    X, W, labels, weight = inputs(T, 1500, 128, seed=T, ignored=ignored)
    check(X, W, labels, weight)
    check(X, W, labels, None, grad=False)
    loss, dX = binding.head_loss(X, W, labels, weight)
    off = labels < 0
    assert not loss[off].any() and not dX[off].any()


@pytest.mark.parametrize("T,V,K,ignored", [(5000, 20000, 64, 0.45), (5000, 20000, 64, 0.7), (5000, 20000, 64, 0.93), (5000, 20000, 1000, 0.99),
                                           (9000, 12000, 72, 0.8), (1900, 40000, 64, 0.6), (3000, 30001, 264, 0.5)])
def test_mostly_ignored(T, V, K, ignored):
    """Where a half, a quarter or an eighth of a chunk counts, two, four or eight pieces of the vocabulary are taken at once."""
    X, W, labels, weight = inputs(T, V, K, seed=T + K, ignored=ignored)
    check(X, W, labels, weight)
    check(X, W, labels, weight, grad=False)


@pytest.mark.parametrize("T", [65536, 65537, 150003])
def test_long_batches(T):
    """More tokens than a gathering CTA counts itself."""
    X, W, labels, weight = inputs(T, 300, 40, seed=T, ignored=0.3)
    check(X, W, labels, weight)
    check(X, W, labels, weight, grad=False)


@pytest.mark.parametrize("T,V,K", [(1810, 29303, 552), (1395, 34181, 952), (4096, 32000, 1000)])
def test_sums_of_any_pitch_over_several_pieces(T, V, K):
    """Copies of the gradient's sums to rows that do not begin on 128 bytes take longer than others; tiles of logits follow them."""
    X, W, labels, weight = inputs(T, V, K, seed=K)
    check(X, W, labels, weight)
    loss, dX = binding.head_loss(X, W, labels, weight)
    for _ in range(4):
        again, dX_again = binding.head_loss(X, W, labels, weight)
        assert torch.equal(again, loss) and torch.equal(dX_again, dX)


@pytest.mark.parametrize("T", [40, 200, 600])
@pytest.mark.parametrize("grad", [True, False])
def test_labels_far_below_the_largest_logit(T, grad):
    """Some rows' references are no good, and the chunk is worked through again."""
    X, W, labels, weight = inputs(T, 3000, 256, seed=5)
    logits = X.float() @ W.float().T
    X = X.clone()
    X[::7] *= 60                                              # logits of +-200, the label's is any of them
    X[3] = -400 * W[labels[3]] + 300 * W[(labels[3] + 1) % 3000]
    far = (X.double() @ W.double().T)
    assert (far.amax(1) - far.gather(1, labels.long()[:, None])[:, 0]).max() > 200 and logits.abs().max() < 60
    check(X, W, labels, weight, grad=grad)


def test_foregone_conclusions():
    """Losses of 1e-5 and below keep their relative precision, and so do their gradients."""
    X, W, labels, weight = inputs(300, 2000, 512, seed=6, sure=60)
    loss, dX = binding.head_loss(X, W, labels, weight)
    want = reference(X, W, labels, weight)[0]
    assert (want < 1e-6).sum() > 50 and (loss > 0).all()
    check(X, W, labels, weight)


def test_repeats_its_bits_and_needs_no_clean_workspace():
    X, W, labels, weight = inputs(1100, 9000, 320, seed=7, ignored=0.3)
    ws = binding.alloc_head_loss_workspace(X, W)
    a = [t.clone() for t in binding.head_loss(X, W, labels, weight, workspace=ws)]
    ws.fill_(255)                                             # NaN in every type
    b = binding.head_loss(X, W, labels, weight, workspace=ws)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_gradient_over_its_input():
    X, W, labels, weight = inputs(333, 4000, 192, seed=8, ignored=0.2)
    kept = X.clone()
    loss, dX = binding.head_loss(X, W, labels, weight, dX=X)
    assert dX.data_ptr() == X.data_ptr()
    want, want_dX, tol, tol_dX = reference(kept, W, labels, weight)
    assert_within(loss, want, tol, "loss")
    assert_within(X, want_dX, tol_dX, "dX")


def test_values_that_are_not_finite_stay_in_their_rows():
    X, W, labels, weight = inputs(300, 1000, 128, seed=9)
    X[5, 3] = float("nan")
    X[9, 0] = float("inf")
    labels[11] = -1
    X[11] = float("nan")
    loss, dX = binding.head_loss(X, W, labels, weight)
    alone, _ = binding.head_loss(X, W, labels, weight, need_grad=False)
    for out in (loss, alone):
        assert not out[[5, 9]].isfinite().any() and out[11] == 0
    assert dX[5].isnan().all() and not dX[9].isfinite().any() and not dX[11].any()
    fine = [i for i in range(300) if i not in (5, 9, 11)]
    want, want_dX, tol, tol_dX = reference(X[fine], W, labels[fine], weight[fine])
    assert_within(loss[fine], want, tol, "loss")
    assert_within(alone[fine], want, tol, "loss alone")
    assert_within(dX[fine], want_dX, tol_dX, "dX")


def test_what_is_refused():
    X, W, labels, weight = inputs(300, 1000, 128, seed=14)
    for grad in (True, False):
        ws = binding.alloc_head_loss_workspace(X, W, grad)
        with pytest.raises(binding.PeqaError) as e:
            binding.head_loss(X, W, labels, weight, need_grad=grad, workspace=ws[:-256])
        assert e.value.status == -5
        with pytest.raises(binding.PeqaError) as e:
            binding.head_loss(X, W, labels, weight, need_grad=grad, workspace=torch.cat([ws, ws])[16:])
        assert e.value.status == -4
    bad = [dict(X=X.float()), dict(X=X[:, :64]), dict(W=W[:, :120].contiguous()), dict(labels=labels.long()), dict(labels=labels[:-1]),
           dict(labels=labels.cpu()), dict(weight=weight[:-1]), dict(weight=weight.double()), dict(loss=torch.empty(299, device="cuda")),
           dict(dX=torch.empty_like(X[:299])), dict(dX=torch.empty_like(X, dtype=torch.float32)), dict(X=X[0]), dict(W=W[0])]
    for more in bad:
        with pytest.raises(ValueError):
            binding.head_loss(**({"X": X, "W": W, "labels": labels, "weight": weight} | more))
    with pytest.raises(binding.PeqaError) as e:
        binding.head_loss(X[:, :100].contiguous(), W[:, :100].contiguous(), labels)
    assert e.value.status == -3
    binding.check_status()


@pytest.mark.parametrize("T", [40, 400])
def test_labels_beyond_the_vocabulary_are_noted(T):
    X, W, labels, weight = inputs(T, 500, 64, seed=10)
    labels[7], labels[8] = 500, 2 ** 31 - 1
    for grad in (False, True):
        loss, dX = binding.head_loss(X, W, labels, weight, need_grad=grad)
        with pytest.raises(binding.PeqaError) as e:
            binding.check_status()
        assert e.value.status == -10
        binding.check_status()
        assert not loss[7:9].any()
    want, want_dX, tol, tol_dX = reference(X, W, labels, weight)
    assert_within(loss, want, tol, "loss")
    assert_within(dX, want_dX, tol_dX, "dX")
    assert not loss[7:9].any() and not dX[7:9].any()


def test_gradient_against_differences():
    """(loss(X + h D) - loss(X - h D)) / 2h along random directions, with losses in 64 bits: off by O(h^2) and bf16's rounding of dX."""
    X, W, labels, _ = inputs(64, 700, 96, seed=11, sure=4)
    _, dX = binding.head_loss(X, W, labels)
    W64 = W.double()
    of = lambda x: torch.nn.functional.cross_entropy(x @ W64.T, labels.long(), reduction="sum")
    for seed in range(4):
        D = torch.randn(X.shape, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        h = 1e-4
        slope = (of(X.double() + h * D) - of(X.double() - h * D)) / (2 * h)
        # bf16's half steps of dX and of the exponentials, over random signs of D: sum of squares, four deviations
        off = 4 * 2.0 ** -8 * 2 * float((dX.double() ** 2).sum()) ** 0.5 + 1e-5
        assert abs(float(slope - (dX.double() * D).sum())) <= off


def test_captured_and_replayed_beside_another_stream():
    X, W, labels, weight = inputs(520, 6000, 256, seed=12, ignored=0.1)
    other = inputs(90, 6000, 256, seed=13)
    want = [t.clone() for t in binding.head_loss(X, W, labels, weight)]
    want_other = [t.clone() for t in binding.head_loss(*other)]
    loss, dX, ws = torch.empty_like(want[0]), torch.empty_like(X), binding.alloc_head_loss_workspace(X, W)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.head_loss(X, W, labels, weight, loss=loss, dX=dX, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        loss.fill_(-1)
        dX.fill_(-1)
        graph.replay()
        with torch.cuda.stream(side):
            got = binding.head_loss(*other)
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(dX, want[1])
        assert torch.equal(got[0], want_other[0]) and torch.equal(got[1], want_other[1])
    # the graph's inputs are read when it runs
    labels[:100] = -1
    graph.replay()
    again = binding.head_loss(X, W, labels, weight)
    assert torch.equal(loss, again[0]) and torch.equal(dX, again[1]) and not loss[:100].any()
