"""The loss of the vocabulary projection in 64 bits, by its definition, and how far binary32 sums of bf16 factors may be from it."""
import torch


def reference(X, W, labels, weight=None):
    """(loss, dX, what the tolerances are made of) in 64 bits, on X's device."""
    T, V = X.shape[0], W.shape[0]
    X64, W64 = X.double(), W.double()
    loss = torch.zeros(T, dtype=torch.float64, device=X.device)
    dX = torch.zeros_like(X64)
    tol_loss, tol_dX = torch.zeros_like(loss), torch.zeros_like(dX)
    g = torch.ones(T, dtype=torch.float64, device=X.device) if weight is None else weight.double()
    live = ((labels >= 0) & (labels < V)).nonzero()[:, 0]
    for rows in live.split(1024):
        at, y = torch.arange(len(rows), device=X.device), labels[rows].long()
        logits = X64[rows] @ W64.T
        rest = logits - logits[at, y][:, None]
        # log of a sum with a 1 in it: where the others come to less than 2^-53 of that, 64 bits show them in log1p alone
        left_out = rest.clone()
        left_out[at, y] = -torch.inf
        total = torch.where(left_out.amax(1) <= 0, torch.log1p(left_out.exp().sum(1)), torch.logsumexp(rest, 1))
        loss[rows] = total
        p = torch.exp(rest - total[:, None])
        others = p.clone()
        others[at, y] = 0
        share = others.sum(1)                                  # 1 - p of the label, without its cancellation
        dX[rows] = (others @ W64 - share[:, None] * W64[y]) * g[rows, None]
        # A logit: a step of the contraction adds 16 products to a binary32 sum and may drop bits below 2^-23 of the sum of
        # magnitudes; so may the label's own, summed elsewhere.
        d = 2 * (X.shape[1] / 16 + 6) * 2.0 ** -23 * (X64[rows].abs() @ W64.abs().T).amax(1)
        # exponential, argument and logarithm: 2^-19 of the sum, with the argument's rounding (2^-24 of up to 100, times log2 e)
        e = d + 2.0 ** -19 + 2.0 ** -23 * rest.abs().amax(1)
        # an exponential below 2^-126 is taken for 0, and there may be one for every entry (3000 of them: 3.5e-35)
        tol_loss[rows] = share * e + 2.0 ** -21 * total.abs() + 2.0 ** -24 * logits.abs().amax(1) * share + V * 2.0 ** -126
        # each exponential is rounded to bf16 (2^-8), the contraction over the vocabulary adds 16 at a time as above
        size = others @ W64.abs() + share[:, None] * W64[y].abs()
        tol_dX[rows] = g[rows, None].abs() * size * (2.0 ** -8 + 2 * e[:, None] + (V / 16 + 6) * 2.0 ** -23) + 2.0 ** -8 * dX[rows].abs() \
            + g[rows, None].abs() * V * 2.0 ** -126 * W64.abs().max()
    return loss, dX, tol_loss, tol_dX


def assert_within(got, want, tol, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values off by more than they may be, the worst " \
                          f"{float((off / tol).nan_to_num(1e9).max()):.2f} times"


def inputs(T, V, K, seed, sure=14.0, ignored=0.0, device="cuda"):
    """Hidden states that lean towards their labels by up to ``sure``, a head of unit gain, labels (a share of them ignored)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=gen, device=device)
    W = (randn(V, K) * K ** -0.5).bfloat16()
    labels = torch.randint(V, (T,), generator=gen, device=device)
    lean = torch.rand((T, 1), generator=gen, device=device) * sure
    X = (randn(T, K) + lean * W[labels].float()).bfloat16()
    if ignored:
        labels = torch.where(torch.rand(T, generator=gen, device=device) < ignored, -100, labels)
    weight = torch.rand(T, generator=gen, device=device) / T
    return X, W, labels.int(), weight
