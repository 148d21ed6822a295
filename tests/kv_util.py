"""Plain forms in 64 bits of the paged cache's operators, on the CPU and by loops over sequences, and what the tests make their
inputs with."""
import math

import numpy as np
import torch

from paper_2305_14152_b200 import binding

BF16_HALF_STEP = 2.0 ** -8          # of a value, relative
H = 2.0 ** -24                      # of binary32


def angles(n_positions, rotary, base=10000.0):
    a = torch.arange(n_positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    return torch.cat([a.cos(), a.sin()], 1).float()


def page_table(lengths, page_size, n_pages, gen, width=None):
    """Pages in no order, each used once; behind a sequence's end the table holds numbers of no page."""
    used = [-(-n // page_size) for n in lengths]
    width = max(1, max(used)) if width is None else width
    order = torch.randperm(n_pages, generator=gen).tolist()
    table, at = torch.full((len(lengths), width), -77, dtype=torch.int32), 0
    table[:, ::2] = 2 ** 30
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table


def places(table, b, positions, page_size):
    pos = torch.as_tensor(list(positions), dtype=torch.long)
    return table[b].long()[pos // page_size], pos % page_size


def quantized(x):
    """Codes and scale per head of binary32 values, every operation in binary32: numpy float32 [..., D]."""
    most = np.abs(x).max(-1)
    scale = np.where(most > 0, most / np.float32(127), np.float32(1)).astype(np.float32)
    return np.rint(x / scale[..., None]).astype(np.int8), scale


def rotated32(x, cos_sin, interleaved):
    """The rotation, every operation in binary32: numpy [tokens, heads, D], cos_sin [tokens, R]."""
    R = cos_sin.shape[1]
    c, s = cos_sin[:, None, :R // 2], cos_sin[:, None, R // 2:]
    y = x.astype(np.float32).copy()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    u, w = y[..., a].copy(), y[..., b].copy()
    y[..., a] = u * c - w * s
    y[..., b] = w * c + u * s
    return y


class Case:
    """A cache whose every place that nobody may read is no number."""

    def __init__(self, seed, lengths, heads, kv_heads, dim, page_size, dtype=torch.bfloat16, order="heads", spare=3, width=None,
                 spread=1.0, window=0):
        self.gen = gen = torch.Generator().manual_seed(seed)
        self.lengths, self.heads, self.kv_heads, self.dim, self.page, self.window = lengths, heads, kv_heads, dim, page_size, window
        n_pages = sum(-(-n // page_size) for n in lengths) + spare
        self.table = page_table(lengths, page_size, n_pages, gen, width)
        shape = (n_pages, page_size, kv_heads, dim)
        self.scales = [None, None]
        self.kv, self.seen = [], torch.zeros(n_pages, page_size, dtype=torch.bool)
        for b, n in enumerate(lengths):
            first = max(0, n - window) if window else 0
            self.seen[places(self.table, b, range(first, n), page_size)] = True
        for i in range(2):
            x = torch.randn(shape, generator=gen) * spread
            if dtype == torch.int8:
                codes, scale = quantized(x.numpy())
                codes, scale = torch.from_numpy(codes), torch.from_numpy(scale)
                codes[~self.seen] = -128                   # a code that is none
                scale[~self.seen] = math.nan
                self.kv.append(codes)
                self.scales[i] = scale.transpose(1, 2).contiguous()
            else:
                x[~self.seen] = math.nan
                self.kv.append(x.to(dtype))
        self.q = (torch.randn(len(lengths), heads, dim, generator=gen) * 1.5).bfloat16()
        self.order = order

    def on_gpu(self):
        def put(x):
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.order == "heads" else x.contiguous().cuda()
        ks, vs = (None if s is None else s.cuda() for s in self.scales)
        return binding.KVCache(put(self.kv[0]), put(self.kv[1]), self.table.cuda(), ks, vs)

    def lens(self):
        return torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def values(self, i, b, first, end):
        """fp64 [tokens, kv_heads, dim]"""
        page, at = places(self.table, b, range(first, end), self.page)
        x = self.kv[i][page, at].double()
        return x if self.scales[i] is None else x * self.scales[i].transpose(1, 2)[page, at].double()[..., None]

    def attention(self, scale=None):
        """out, lse, and how far off a kernel may be from each: fp64."""
        B, D, G = len(self.lengths), self.dim, self.heads // self.kv_heads
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        out, lse = torch.zeros(B, self.heads, D, dtype=torch.float64), torch.full((B, self.heads), -math.inf, dtype=torch.float64)
        out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
        for b, n in enumerate(self.lengths):
            first = max(0, n - self.window) if self.window else 0
            if n == first:
                continue
            k, v = self.values(0, b, first, n), self.values(1, b, first, n)
            q = self.q[b].double().view(self.kv_heads, G, D)
            s = torch.einsum("kgd,tkd->kgt", q, k) * scale
            total = torch.logsumexp(s, -1)
            p = torch.exp(s - total[..., None])
            # What a score may be off by.  D products, exact in binary32 (16-bit factors; a key's scale comes behind the sum), whose sum
            # loses at most 2 h per addition (a tensor core may cut what is below the last bit instead of rounding), then
            # four roundings of the score: D * 2 h of the sum of the products' sizes, 4 h of the score.  8-bit caches: q in binary16 with a
            # common power of two is off by 2^-25 of the head's largest at most, 2^-25 D |q|max |k|max in all; and a code c is summed as c + 128,
            # the sum of 128 q taken off afterwards, so that the products are of the size of q (|c| + 128) and once more 128 q.
            sizes = k.abs()
            if self.scales[0] is not None:
                page, at = places(self.table, b, range(first, n), self.page)
                sizes = sizes + 256 * self.scales[0].transpose(1, 2)[page, at].double()[..., None]
            size = torch.einsum("kgd,tkd->kgt", q.abs(), sizes) * abs(scale)
            ds = 2 * H * D * size + 4 * H * s.abs()
            if self.scales[0] is not None:
                ds = ds + 2.0 ** -25 * D * abs(scale) * q.abs().amax(-1)[..., None] * k.abs().amax(-1).t()[:, None, :]
            off = (p * torch.expm1(ds)).nan_to_num(nan=0.0)   # a token whose p is 0 has no part, however far off its score is
            # exp2 (2 ulp, and the rounding of its argument, whose size is below 2^7 where p matters: 2^7 h ln 2 of p), p as two numbers of 8
            # and more bits (2^-17 of p), n additions of p and of p v, a few roundings where parts are joined; numerator and denominator both.
            rel = 2 * (100 * H + 2.0 ** -16 + 2 * H * (n + 64))
            spread = torch.einsum("kgt,tkd->kgd", p, v.abs())
            o = torch.einsum("kgt,tkd->kgd", p, v)
            out[b], lse[b] = o.reshape(-1, D), total.reshape(-1)
            inner = torch.einsum("kgt,tkd->kgd", off, v.abs()) + (off.sum(-1)[..., None] + rel) * spread
            if self.scales[1] is not None:
                # p times the scale of its value is a binary16 number in units of 2^-6 of the row's largest scale: off by half a step, 2^-11 of it, or
                # by half of the smallest, 2^-25, whatever p is.  p is relative to the largest score or to one that was up to 2^8 smaller,
                # which only makes it larger.  So 2^-31 of the largest scale per code, over the sum of p relative to the largest.
                inner = inner + 2.0 ** -11 * spread
                page, at = places(self.table, b, range(first, n), self.page)
                most = self.scales[1].transpose(1, 2)[page, at].double().abs().amax(0)             # [kv_heads]
                codes = self.kv[1][page, at].double().abs().sum(0)                                 # [kv_heads, dim]
                inner = inner + 2.0 ** -31 * (most[:, None] * codes)[:, None, :] * p.amax(-1)[..., None]
            out_tol[b] = (BF16_HALF_STEP * (o.abs() + inner) + inner).reshape(-1, D) + 1e-37
            lse_tol[b] = (off.sum(-1) + rel + 4 * H * total.abs()).reshape(-1)
        return out, lse, out_tol, lse_tol


def assert_within(got, ref, tol, what):
    got = got.detach().double().cpu()
    same = (got == ref)                                    # infinities
    bad = ~same & ~((got - ref).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, at {bad.nonzero()[0].tolist()}: " \
        f"{got[bad][0]} for {ref[bad][0]}, {tol[bad][0]} allowed"
