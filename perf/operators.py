"""Attention of token generation over a paged key-value cache, beside the quantized linears of a layer.

Between the q, k and v projections of a decoder layer and its output projection a generation step rotates the new
queries and keys by their positions, appends keys and values to the cache, and lets every new token attend to the
cache of its sequence.  Two operators do that; a case names one of them (``op``) and its sizes:

  append  q and k rotated by the angles of their positions; k and v written to their places in the cache.  ``new`` tokens in all,
          one per sequence (``ragged`` false: generation) or split unevenly over the sequences (true: prompts, or the
          next piece of each).
  attend  softmax(q k^T scale) v of one new token per sequence over its cached tokens; with ``window`` over the last so many.

``seqs`` sequences of up to ``length`` tokens, ``heads`` query heads that share ``kv_heads`` key-value heads of ``dim``
channels; pages of ``page`` tokens; ``cache`` "bf16", or "int8" (codes with one scale per token and head); ``order`` says
whether a page keeps the tokens of one head together ("heads") or the heads of one token ("tokens").  ``holes``: every
eighth sequence is empty, as in a batch padded to a fixed size.
"""
import math

import torch

own = False


def _case(name, op, seqs, length, new, ragged, heads, kv_heads, dim, page, cache, order, window=0, holes=False):
    named = {} if name is None else {"name": name}
    return named | {"op": op, "seqs": seqs, "length": length, "new": new, "ragged": ragged, "heads": heads,
                    "kv_heads": kv_heads, "dim": dim, "page": page, "cache": cache, "order": order, "window": window, "holes": holes}


def listed():
    return [
        # one sequence generated on a layer as wide as LLaMA-7B's (4096 = 32 heads of 128): the latency of a chat server
        _case("append_1_token", "append", 1, 129, 1, False, 32, 32, 128, 16, "bf16", "heads"),
        # a full serving batch on a layer as wide as LLaMA-65B's (8192 = 64 heads of 128), the cache in 8 bits
        _case("append_16_tokens_int8", "append", 16, 1001, 16, False, 64, 64, 128, 16, "int8", "heads"),
        # a large batch with grouped heads, padded to its fixed size
        _case("append_256_tokens_grouped", "append", 256, 700, 256, False, 64, 8, 128, 32, "bf16", "tokens", holes=True),
        # prompts of uneven lengths, 4096 tokens in all: the token count of a training step of the benchmark
        _case("append_prompts", "append", 7, 1301, 4096, True, 64, 64, 128, 16, "bf16", "heads"),
        # the next pieces of long prompts into an 8-bit cache
        _case("append_pieces_int8", "append", 5, 2100, 2048, True, 32, 32, 128, 64, "int8", "tokens"),
        # the smallest call: a chat that has just begun
        _case("attend_short", "attend", 1, 129, 1, False, 32, 32, 128, 16, "bf16", "heads"),
        # a full serving batch on a layer as wide as LLaMA-65B's, contexts of up to 4000 tokens: an ordinary step
        _case("attend_16_seqs", "attend", 16, 4001, 16, False, 64, 64, 128, 16, "bf16", "heads"),
        # one long document with grouped heads
        _case("attend_long", "attend", 1, 131071, 1, False, 64, 8, 128, 64, "bf16", "heads"),
        # a large batch with grouped heads, its cache in 8 bits and padded to its fixed size
        _case("attend_64_seqs_int8", "attend", 64, 8190, 64, False, 64, 8, 128, 16, "int8", "heads", holes=True),
        # the largest: long contexts, a head of keys and values for each query head, 8 bits
        _case("attend_4_long_int8", "attend", 4, 32003, 4, False, 64, 64, 128, 32, "int8", "tokens"),
        # many short chats at once
        _case("attend_256_short", "attend", 256, 513, 256, False, 32, 32, 128, 16, "bf16", "tokens"),
        # attention to the last 1024 tokens alone, heads of 64 channels
        _case("attend_window", "attend", 24, 6000, 24, False, 32, 4, 64, 16, "bf16", "heads", window=1024),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: query heads and key-value heads: one for each, groups of 2 to 16, and one key-value head for all
_HEADS = [(8, 8), (16, 1), (20, 4), (28, 4), (32, 2), (32, 4), (32, 8), (32, 32), (40, 40), (52, 52), (64, 8), (64, 64), (71, 1)]


def draw(rng):
    heads, kv_heads = rng.choice(_HEADS)
    dim = rng.choice([64, 128, 128, 128, 256])
    op = rng.choice(["append", "attend"])
    cache, order = rng.choice(["bf16", "int8"]), rng.choice(["heads", "tokens"])
    page = rng.choice([8, 16, 16, 32, 48, 64, 128])
    if op == "append":
        ragged = rng.random() < 0.5
        seqs = _log_uniform(rng, 1, 16 if ragged else 256)
        most = max(seqs + 1, min(4096, (4096 * 192 * 128) // ((heads + 2 * kv_heads) * dim)))
        new = _log_uniform(rng, seqs, most) if ragged else seqs
        length = -(-2 * new // seqs) + rng.randrange(1, 600) if ragged else _log_uniform(rng, 1, 1000)
        return _case(None, op, seqs, length, new, ragged, heads, kv_heads, dim, page, cache, order, 0, rng.random() < 0.3)
    seqs = _log_uniform(rng, 1, 256)
    most = max(2, min(131072, (4 * 32003 * 64 * 128) // (seqs * max(kv_heads, heads // 16) * dim * (2 if cache == "bf16" else 1))))
    length = _log_uniform(rng, 1, most)
    window = _log_uniform(rng, 1, length) if rng.random() < 0.25 else 0
    return _case(None, op, seqs, length, seqs, False, heads, kv_heads, dim, page, cache, order, window, rng.random() < 0.3)


def _spread(n, lo, hi):
    """n whole numbers of [lo, hi], evenly spread and in no order (the golden section's multiples); the first is hi."""
    return [hi - int((hi - lo + 1) * ((i * 0.6180339887498949) % 1.0)) if hi > lo else hi for i in range(n)]


def _new_tokens(case):
    """New tokens of every sequence."""
    n = case["seqs"]
    if not case["ragged"]:
        return [0 if case["holes"] and i % 8 == 5 else 1 for i in range(n)]
    share = [1 + w for w in _spread(n, 0, 99)]
    spare = case["new"] - n
    counts = [1 + spare * w // sum(share) for w in share]
    counts[-1] += case["new"] - sum(counts)
    return counts


def _lengths(case):
    """Tokens of every sequence with the new ones, 0 for one that is not there."""
    return [max(t, l) if t else 0 for t, l in zip(_new_tokens(case), _spread(case["seqs"], -(-case["length"] // 4), case["length"]))]


def _positions(case):
    return max(1, max(_lengths(case)))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    B, H, D, page = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    lengths, counts = _lengths(case), _new_tokens(case)
    ints = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")
    width = -(-max(1, max(lengths)) // page)                       # pages of the longest sequence
    used = [-(-l // page) for l in lengths]
    n_pages = sum(used) + 3
    shuffled = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    # a page table has something in every place; behind a sequence's end it means nothing
    rows = torch.arange(width, device="cuda")[None, :]
    first = torch.tensor([sum(used[:i]) for i in range(B)], device="cuda")[:, None]
    there = rows < torch.tensor(used, device="cuda")[:, None]
    table = torch.where(there, shuffled[torch.where(there, first + rows, 0)], 0).to(torch.int32).contiguous()
    s = {"case": case, "table": table, "lengths": ints(lengths), "page": page, "scale": 1.0 / math.sqrt(D), "window": case["window"]}

    def cache():
        shape = (n_pages, H, page, D) if case["order"] == "heads" else (n_pages, page, H, D)
        x = randn(*shape)
        scales = None
        if case["cache"] == "int8":
            x = x.float()
            scales = (x.abs().amax(-1) / 127).clamp_min(1e-30)
            x = torch.round(x / scales[..., None]).to(torch.int8)
            scales = (scales if case["order"] == "heads" else scales.transpose(1, 2)).contiguous()   # [n_pages, H, page]
        return (x.transpose(1, 2) if case["order"] == "heads" else x), scales                       # [n_pages, page, H, D]

    s["k"], s["k_scales"] = cache()
    s["v"], s["v_scales"] = cache()
    if case["op"] == "attend":
        s["q"] = 2 * randn(B, case["heads"], D)
        return s
    # q, k and v as one projection leaves them, side by side in the rows of one matrix; a padded batch has a row for every place
    T = case["new"]
    qkv = randn(T, case["heads"] + 2 * H, D)
    s["q"], s["new_k"], s["new_v"] = qkv.split([case["heads"], H, H], dim=1)
    s["starts"] = ints([sum(counts[:i]) for i in range(B + 1)]) if case["ragged"] else None
    s["q_out"] = torch.zeros((T, case["heads"], D), dtype=torch.bfloat16, device="cuda")
    # cos and sin of position * 10000^(-2i/D), taken in 64 bits
    angles = torch.arange(_positions(case), device="cuda", dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    s["cos_sin"] = torch.cat([angles.cos(), angles.sin()], 1).float()
    return s


def _handle(s):
    """The framework's descriptor of the cache, and the scratch of its attention: made once, as a program would."""
    if "handle" not in s:
        from paper_2305_14152_b200 import binding
        s["binding"] = binding
        s["handle"] = binding.KVCache(s["k"], s["v"], s["table"], s["k_scales"], s["v_scales"])
        s["workspace"] = binding.alloc_attn_workspace(s["handle"], s["case"]["heads"])
    return s["binding"], s["handle"]


def _places(s):
    """Sequence, position, page and place in the page of every new token that has one."""
    T, lengths = s["q"].shape[0], s["lengths"].long()
    t = torch.arange(T, device="cuda")
    if s["starts"] is None:
        seq, pos = t, lengths - 1
    else:
        starts = s["starts"].long()
        seq = torch.searchsorted(starts, t, right=True) - 1
        pos = lengths[seq] - starts[seq + 1] + t
    live = (pos >= 0).nonzero()[:, 0] if s["case"]["holes"] else t
    seq, pos = seq[live], pos[live]
    return live, pos, s["table"].long()[seq, pos // s["page"]], pos % s["page"]


def _rotated(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(s):
    live, pos, page, at = _places(s)
    cos, sin = s["cos_sin"][pos][:, None, :].chunk(2, -1)
    s["q_out"][live] = _rotated(s["q"][live], cos, sin).bfloat16()
    for x, cache, scales in ((_rotated(s["new_k"][live], cos, sin), s["k"], s["k_scales"]), (s["new_v"][live].float(), s["v"], s["v_scales"])):
        if scales is not None:
            most = x.abs().amax(-1)
            step = torch.where(most > 0, most / torch.full_like(most, 127), torch.ones_like(most))
            scales[page, :, at] = step
            x = torch.round(x / step[..., None])
        cache[page, at] = x.to(cache.dtype)
    return _append_outputs(s)


def _append_outputs(s):
    # the codes of an 8-bit cache as they are: whole numbers, which nothing but equal is right for, and their scales
    kept = [s["q_out"], s["k"], s["v"]]
    return kept + [s["k_scales"], s["v_scales"]] if s["k_scales"] is not None else kept


def _cached(s, cache, scales):
    """[seqs, kv_heads, tokens of the table's width, dim]"""
    x = cache[s["table"].long()].float()                           # [seqs, pages, page, kv_heads, dim]
    if scales is not None:
        x *= scales[s["table"].long()].transpose(2, 3)[..., None]
    B, P, page, H, D = x.shape
    return x.reshape(B, P * page, H, D).transpose(1, 2)


def _attend(s):
    B, heads, D = s["q"].shape
    k = _cached(s, s["k"], s["k_scales"])
    H, width = k.shape[1:3]
    scores = s["q"].float().view(B, H, heads // H, D) @ k.transpose(2, 3) * s["scale"]
    del k
    lengths, t = s["lengths"].long()[:, None], torch.arange(width, device="cuda")[None, :]
    seen = t < lengths
    if s["window"]:
        seen &= t >= lengths - s["window"]
    scores = scores.masked_fill(~seen[:, None, None, :], -math.inf)
    most = scores.amax(-1, keepdim=True).clamp_min(-3.0e38)        # finite where nothing is seen
    p = torch.exp(scores - most)
    total = p.sum(-1, keepdim=True)
    v = _cached(s, s["v"], s["v_scales"])
    v = v.masked_fill(~seen[:, None, :, None], 0.0)                # what lies behind a sequence's end is no number to rely on
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.where(total > 0, most + torch.log(total), torch.full_like(total, -math.inf))
    return out.view(B, heads, D).bfloat16(), lse.view(B, heads)


def run(s):
    if s["case"]["op"] == "append":
        if not own:
            return _append(s)
        binding, cache = _handle(s)
        binding.kv_append(cache, s["q"], s["new_k"], s["new_v"], s["cos_sin"], s["lengths"], s["starts"], q_out=s["q_out"])
        return _append_outputs(s)
    if not own:
        return _attend(s)
    binding, cache = _handle(s)
    return binding.attn_decode(cache, s["q"], s["lengths"], window=s["window"], workspace=s["workspace"], return_lse=True)


def work(case):
    heads, H, D = case["heads"], case["kv_heads"], case["dim"]
    size, scale = (2, 0) if case["cache"] == "bf16" else (1, 4)
    counts, lengths = _new_tokens(case), _lengths(case)
    if case["op"] == "append":
        T = sum(counts)
        rows = T * (2 * 2 * heads * D + 2 * H * (2 * D + size * D + scale))
        angles = 4 * D * len({l - i for c, l in zip(counts, lengths) for i in range(1, c + 1)})
        return {"bytes": rows + angles + 4 * 2 * case["seqs"] + 4 * T, "flops": 3 * T * (heads + H) * D}
    seen = [min(l, case["window"]) if case["window"] else l for l in lengths]
    tokens, live = sum(seen), sum(1 for l in seen if l)
    pages = sum(-(-l // case["page"]) for l in seen)
    return {"bytes": tokens * 2 * H * (size * D + scale) + live * 2 * heads * D + case["seqs"] * heads * (2 * D + 4) + 4 * (pages + case["seqs"]),
            "flops": 4 * tokens * heads * D}


def exact(case, seed):
    s = prepare(case, seed)
    lengths, table = _lengths(case), s["table"].tolist()
    page, D, G = case["page"], case["dim"], case["heads"] // case["kv_heads"]
    if case["op"] == "append":
        q_out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
        ks, vs = (None, None) if s["k_scales"] is None else (s["k_scales"].double(), s["v_scales"].double())
        at = 0
        for b, count in enumerate(_new_tokens(case)):
            rows = torch.arange(at, at + count, device="cuda") if case["ragged"] else torch.full((count,), b, device="cuda")
            at += count
            if not count:
                continue
            pos = torch.arange(lengths[b] - count, lengths[b], device="cuda")
            cos, sin = s["cos_sin"][pos, None, :D // 2].double(), s["cos_sin"][pos, None, D // 2:].double()
            turn = lambda x: torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin, x[..., D // 2:] * cos + x[..., :D // 2] * sin], -1)
            where = (torch.tensor(table[b], device="cuda")[pos // page], pos % page)
            new_k, new_v = turn(s["new_k"][rows].double()), s["new_v"][rows].double()
            q_out[rows] = turn(s["q"][rows].double())
            if ks is None:
                k[where], v[where] = new_k, new_v
            else:
                ks[where[0], :, where[1]], vs[where[0], :, where[1]] = new_k.abs().amax(-1) / 127, new_v.abs().amax(-1) / 127
        # a code is a decision taken in 32 bits (value / scale, rounded): it has no value in 64
        return [q_out, k, v] if ks is None else [q_out, None, None, ks, vs]
    out = torch.zeros((case["seqs"], case["heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((case["seqs"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == first:
            continue
        t = torch.arange(first, n, device="cuda")
        pages = torch.tensor(table[b], device="cuda")[t // page]

        def of(cache, scales):
            x = cache[pages, t % page].double()                    # [tokens, kv_heads, dim]
            return x if scales is None else x * scales[pages, :, t % page].double()[..., None]

        q = s["q"][b].double().view(-1, G, D)
        scores = torch.einsum("kgd,tkd->kgt", q, of(s["k"], s["k_scales"])) / math.sqrt(D)
        total = torch.logsumexp(scores, -1)
        lse[b] = total.reshape(-1)
        out[b] = torch.einsum("kgt,tkd->kgd", torch.exp(scores - total[..., None]), of(s["v"], s["v_scales"])).reshape(-1, D)
    return out, lse
