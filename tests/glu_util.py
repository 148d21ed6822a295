"""The gated block in 64 bits, by its definition, and how far the kernels' sums may be from it."""
import math

import torch

from paper_2305_14152_b200 import binding


def block(F, K, bits, group, seed, device="cuda"):
    """A gated block of random codes, as wide scales as a matrix of unit gain has, and its weights s (Q - z) in 64 bits."""
    gen = torch.Generator(device=device).manual_seed(seed)
    N, G = 2 * F, 1 if group in (0, K) else K // group
    codes = torch.randint(2 ** bits, (N, K), generator=gen, device=device).to(torch.uint8)
    zeros = torch.randint(2 ** bits, (N, G), generator=gen, device=device).to(torch.uint8)
    scales = (0.5 + torch.rand((N, G), generator=gen, device=device)) * K ** -0.5 * 3.5 / 2 ** bits
    w = binding.QWeight(bits, N, K, group, binding.pack(codes, bits), zeros, scales)
    return w, weights(codes, zeros, scales), codes


def weights(codes, zeros, scales):
    N, K = codes.shape
    G = zeros.shape[1]
    return ((codes.double().view(N, G, K // G) - zeros.double()[:, :, None]) * scales.double()[:, :, None]).view(N, K)


def halves(y):
    """Gate and up side of [tokens, 2F]."""
    y = y.unflatten(1, (-1, 2, 8))
    return y[:, :, 0].flatten(1), y[:, :, 1].flatten(1)


def act(x, activation):
    if activation == "silu":
        return x * torch.sigmoid(x)
    # (1 + tanh(u)) / 2 as the logistic function of 2u: 64 bits of 1 + tanh(-18) are all rounding
    return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))


def forward(X, W, activation, folded):
    """(H, Y, tolerances of both).  folded: the operand is (Q - z) s in binary16 (groups of columns); else codes are exact."""
    X64 = X.double()
    Y = X64 @ W.T
    K = X.shape[1]
    size = X64.abs() @ W.abs().T
    # two half steps of binary16 where scales are folded in, in units that the row's largest follows; a binary32 sum of 16 products at a time, which
    # may drop what is below 2^-23 of the sum of magnitudes; the scale's own product; activations are rounded at 2^-25 of the row's largest
    d = size * ((2 * 2.0 ** -11 if folded else 0.0) + (K / 16 + 6) * 2.0 ** -23) \
        + 2.0 ** -25 * X64.abs().amax(1, keepdim=True) * W.abs().sum(1)[None]
    if folded:
        d = d + 2.0 ** -24 * X64.abs().sum(1, keepdim=True) * W.abs().amax(1)[None]
    gate, up = halves(Y)
    dg, du = halves(d)
    a = act(gate, activation)
    H = a * up
    # slopes of both activations lie within 1.13; the activation itself is good to 2^-18
    tol = 1.13 * dg * (up.abs() + du) + a.abs() * du + (2.0 ** -8 + 2.0 ** -18) * (a.abs() + 1.13 * dg) * (up.abs() + du)
    return H, Y, tol, d + 2.0 ** -8 * (Y.abs() + d)


def backward(Y, dH, activation):
    """(dY, tolerance) of Y and dH as they are."""
    x = Y.double().requires_grad_()
    gate, up = halves(x)
    (act(gate, activation) * up * dH.double()).sum().backward()
    dY = x.grad
    gate, up = (t.detach() for t in (gate, up))
    # binary32 terms: each good to 2^-18 of itself; those of the gate's slope may cancel
    c, k = 2 * math.sqrt(2 / math.pi), 0.044715
    v, slope = (gate, torch.ones_like(gate)) if activation == "silu" else (c * (gate + k * gate ** 3), c * (1 + 3 * k * gate ** 2))
    p, q = torch.sigmoid(v), torch.sigmoid(-v)
    terms = torch.stack([((dH.double() * up).abs() * (p + (gate * p * q * slope).abs())).unflatten(1, (-1, 8)),
                         (dH.double() * gate * p).abs().unflatten(1, (-1, 8))], 2).flatten(1)
    # (1 + |v|) times the rounding of v, which the exponential takes over
    worse = torch.stack([(1 + v.abs()).clamp(max=200).unflatten(1, (-1, 8))] * 2, 2).flatten(1)
    return dY, 2.0 ** -8 * dY.abs() + terms * (2.0 ** -18 + 4 * 2.0 ** -24 * worse) + 2.0 ** -126
